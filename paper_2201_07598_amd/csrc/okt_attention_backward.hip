// okt_attention_backward: the gradients, with the probabilities taken again from q, k and
// the log-sum-exp.
//
// Two kernels, each of which keeps what it sums in registers, so nothing is added across
// workgroups and the result does not change from run to run:
//   queries  a wave owns 32 queries and passes over the keys: S' = K Q', dP' = V dO' (keys
//            down, queries across), dQ' += K' dS'; it also takes D = dO . O of its rows
//   keys     a wave owns 32 keys and passes over the queries of every head of the group:
//            S = Q K', dP = dO V' (queries down, keys across), dV' += dO' P, dK' += Q' dS
// The scores and dP are formed twice, 7 products where 5 would do: the alternative adds dQ in
// memory from every key block, in an order that changes from run to run.
#include "okt_attention.h"

namespace okt {

constexpr int BWD_THREADS = 256;
constexpr int BWD_ROWS = BWD_THREADS / WAVE * 32;     // queries or keys of a workgroup
constexpr int BWD_TILE = 64;                          // keys or queries that pass by together

// log-sum-exp to base 2, +inf for a row that sees nothing: its probabilities come out as 0
__device__ __forceinline__ float lse_log2(float lse) { return lse == -INFINITY ? INFINITY : lse * 1.44269504088896f; }

template <typename T, int DIM, bool DROP>
__global__ __launch_bounds__(BWD_THREADS, DIM == 64 ? 2 : 1) void attention_backward_queries_kernel(
    AttentionArgs a, const T* q, const T* k, const T* v, const T* o, const float* lse, const T* d_o, T* dq, float* rows_d,
    uint32_t blocks) {
    using Tile = RowTile<T, DIM, BWD_TILE, BWD_THREADS>;
    __shared__ __attribute__((aligned(1024))) char shared[4 * Tile::BYTES];
    const uint32_t place = near_place(blockIdx.x, gridDim.x), plane = place / blocks;
    const uint32_t b = plane / a.heads, h = plane % a.heads, kv = h / a.group;
    const uint32_t wave = uniform(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const int ql = sequence_length(a.q_lens, b, a.q_len), kl = sequence_length(a.k_lens, b, a.k_len);
    const int q0 = (blocks - 1 - place % blocks) * BWD_ROWS, w0 = q0 + 32 * (int)wave, i = w0 + (int)(lane % 32);
    const int past = kl - ql + 1;
    const auto seen = [&](int query) { const int n = query + past; return query >= ql ? 0 : !a.causal || n > kl ? kl : n < 0 ? 0 : n; };
    const int keys = q0 < ql ? seen(q0 + BWD_ROWS < ql ? q0 + BWD_ROWS - 1 : ql - 1) : 0;
    const int mine = seen(i), wave_least = w0 + 31 < ql ? seen(w0) : 0;
    const int wave_most = w0 < ql ? seen(w0 + 32 < ql ? w0 + 31 : ql - 1) : 0;

    f32x16 acc[DIM / 32];
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) acc[d] = 0.0f;
    if (keys > 0) {
        const T* kb = k + b * a.k.batch + kv * a.k.head;
        const T* vb = v + b * a.v.batch + kv * a.v.head;
        const uint64_t row = i < ql ? i : ql - 1;
        const T* q_row = q + b * a.q.batch + row * a.q.row + h * a.q.head;
        const T* do_row = d_o + b * a.d_o.batch + row * a.d_o.row + h * a.d_o.head;
        const T* o_row = o + b * a.o.batch + row * a.o.row + h * a.o.head;
        const uint32_t k_row = (uint32_t)a.k.row * 2, v_row = (uint32_t)a.v.row * 2;
        const typename Tile::Places k_at(k_row, a.head_dim), v_at(v_row, a.head_dim);
        const uint32_t lds = lds_address(shared);
        Tile::fetch(lds, kb, k_row, k_at, 0, 0, kl, a.head_dim);
        Tile::fetch(lds + Tile::BYTES, vb, v_row, v_at, 0, 0, kl, a.head_dim);
        frag<T> qf[DIM / 16], df[DIM / 16];
        float sum = 0.0f;
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            qf[s] = row_operand(q_row, s, a.head_dim);
            df[s] = row_operand(do_row, s, a.head_dim);
            const f32x8 x = __builtin_convertvector(df[s], f32x8), y = __builtin_convertvector(row_operand(o_row, s, a.head_dim), f32x8);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], y[e], sum);
        }
        sum = sum_halves(sum);
        const float base = lse_log2(lse[(uint64_t)plane * a.q_len + row]);
        RandomKey key = {0, 0};
        if (DROP) key = random_key(a.seed);

        for (int key0 = 0, turn = 0; key0 < keys; key0 += BWD_TILE, turn ^= 1) {
            fetched();
            const char* kt = shared + turn * 2 * Tile::BYTES;
            const char* vt = kt + Tile::BYTES;
            if (key0 + BWD_TILE < keys) {
                const uint32_t next = lds + (turn ^ 1) * 2 * Tile::BYTES;
                Tile::fetch(next, kb, k_row, k_at, key0 + BWD_TILE, 0, kl, a.head_dim);
                Tile::fetch(next + Tile::BYTES, vb, v_row, v_at, key0 + BWD_TILE, 0, kl, a.head_dim);
            }
            if (key0 >= wave_most) continue;
            const bool masked = key0 + BWD_TILE > wave_least;
#pragma unroll
            for (int n = 0; n < BWD_TILE / 32; ++n) {
                f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) s = mfma(Tile::rows(kt, 32 * n, e), qf[e], s);
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) dp = mfma(Tile::rows(vt, 32 * n, e), df[e], dp);
                if (DROP) {
                    uint32_t w[16];
                    kept_keys(w, i, key0 + 32 * n, plane, key, a.site);
                    const uint32_t mask = lane & 1 ? 0xffffffffu : 0xffffu, bar = a.drop.bar << (16 * (lane & 1));
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[r] = (w[r] & mask) < bar ? dp[r] * a.drop.scale : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -base));
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = key0 + 32 * n + 16 * (int)(lane / 32) + r < mine ? s[r] : 0.0f;
                }
                if (n == 0 && key0 == 0) {
                    // A row that sees no key past this tile takes D from what it has here, sum_j p dP: few
                    // probabilities are large ones, and the rounding of o would show in dP - D.
                    float few = 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) few = __builtin_fmaf(s[r], dp[r], few);
                    few = sum_halves(few);
                    sum = mine <= 32 ? few : sum;
                    if (lane < 32 && i < ql) rows_d[(uint64_t)plane * a.q_len + i] = sum;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] *= dp[r] - sum;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const frag<T> ds = to_operand<T>(s, t);
#pragma unroll
                    for (int d = 0; d < DIM / 32; ++d) acc[d] = mfma(Tile::columns(kt, 32 * n, d, t), ds, acc[d]);
                }
            }
        }
    }
    if (i < (int)a.q_len) {
        T* out = dq + b * a.dq.batch + (uint64_t)i * a.dq.row + h * a.dq.head;
        if (mine == 0) {
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d) acc[d] = 0.0f;
        }
        store_row(out, acc, a.scale, a.head_dim);
    }
}

template <typename T, int DIM, bool DROP>
__global__ __launch_bounds__(BWD_THREADS, DIM == 64 ? 2 : 1) void attention_backward_keys_kernel(
    AttentionArgs a, const T* q, const T* k, const T* v, const float* lse, const T* d_o, const float* rows_d, T* dk, T* dv,
    uint32_t blocks) {
    using Tile = RowTile<T, DIM, BWD_TILE, BWD_THREADS>;
    __shared__ __attribute__((aligned(1024))) char shared[4 * Tile::BYTES];
    __shared__ float2 rows_of[2][BWD_TILE];                    // log-sum-exp and D of the tile's rows
    const uint32_t place = near_place(blockIdx.x, gridDim.x), b = place / blocks / a.kv_heads, kv = place / blocks % a.kv_heads;
    const uint32_t wave = uniform(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const int ql = sequence_length(a.q_lens, b, a.q_len), kl = sequence_length(a.k_lens, b, a.k_len);
    const int k0 = place % blocks * BWD_ROWS, w0 = k0 + 32 * (int)wave, j = w0 + (int)(lane % 32);
    // the first query that sees key j, and the first that sees any
    const auto first_for = [&](int key) { const int n = a.causal ? key - (kl - ql) : 0; return n < 0 ? 0 : n; };
    const int lo = first_for(0), begin = first_for(k0) / BWD_TILE * BWD_TILE;
    const int mine = j < kl ? first_for(j) : ql;
    const int wave_least = w0 < kl ? first_for(w0) : ql + BWD_TILE, wave_most = w0 + 31 < kl ? first_for(w0 + 31) : ql;
    const int tiles = k0 < kl && begin < ql ? (ql - begin + BWD_TILE - 1) / BWD_TILE : 0;

    f32x16 dkacc[DIM / 32], dvacc[DIM / 32];
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) dkacc[d] = dvacc[d] = 0.0f;
    if (tiles > 0) {
        const uint64_t row = j < kl ? j : kl - 1;
        const T* k_row = k + b * a.k.batch + row * a.k.row + kv * a.k.head;
        const T* v_row = v + b * a.v.batch + row * a.v.row + kv * a.v.head;
        frag<T> kf[DIM / 16], vf[DIM / 16];
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            kf[s] = row_operand(k_row, s, a.head_dim);
            vf[s] = row_operand(v_row, s, a.head_dim);
        }
        RandomKey key = {0, 0};
        if (DROP) key = random_key(a.seed);
        const uint32_t q_row = (uint32_t)a.q.row * 2, do_row = (uint32_t)a.d_o.row * 2, lds = lds_address(shared);
        const typename Tile::Places q_at(q_row, a.head_dim), do_at(do_row, a.head_dim);
        const auto fetch = [&](int it, int turn) {
            const uint32_t h = kv * a.group + it / tiles;
            const int first = begin + it % tiles * BWD_TILE;
            const uint32_t to = lds + turn * 2 * Tile::BYTES;
            Tile::fetch(to, q + b * a.q.batch + h * a.q.head, q_row, q_at, first, lo, ql, a.head_dim);
            Tile::fetch(to + Tile::BYTES, d_o + b * a.d_o.batch + h * a.d_o.head, do_row, do_at, first, lo, ql, a.head_dim);
            if (threadIdx.x < BWD_TILE) {
                const int i = first + (int)threadIdx.x;
                const uint64_t at = ((uint64_t)b * a.heads + h) * a.q_len + (i < lo ? lo : i > ql - 1 ? ql - 1 : i);
                rows_of[turn][threadIdx.x] = make_float2(lse_log2(lse[at]), rows_d[at]);
            }
        };
        fetch(0, 0);
        const int steps = tiles * (int)a.group;
        for (int it = 0, turn = 0; it < steps; ++it, turn ^= 1) {
            fetched();
            const char* qt = shared + turn * 2 * Tile::BYTES;
            const char* dt = qt + Tile::BYTES;
            if (it + 1 < steps) fetch(it + 1, turn ^ 1);
            const uint32_t plane = b * a.heads + kv * a.group + it / tiles;
            const int query0 = begin + it % tiles * BWD_TILE;
            if (query0 + BWD_TILE <= wave_least) continue;
            const bool masked = query0 < wave_most || query0 + BWD_TILE > ql;
#pragma unroll
            for (int n = 0; n < BWD_TILE / 32; ++n) {
                f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) s = mfma(Tile::rows(qt, 32 * n, e), kf[e], s);
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) dp = mfma(Tile::rows(dt, 32 * n, e), vf[e], dp);
                uint32_t w[8];
                if (DROP) kept_queries(w, j, query0 + 32 * n, plane, key, a.site);
                const int at = 32 * n + 16 * (int)(lane / 32);
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float2 ld = rows_of[turn][at + r];
                    const int i = query0 + at + r;
                    float p = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -ld.x));
                    if (masked) p = i >= mine && i < ql ? p : 0.0f;
                    float d = dp[r];
                    s[r] = p;
                    if (DROP) {
                        const bool keep = r & 1 ? w[r / 2] < a.drop.bar << 16 : (w[r / 2] & 0xffffu) < a.drop.bar;
                        d = keep ? d * a.drop.scale : 0.0f;
                        s[r] = keep ? p * a.drop.scale : 0.0f;
                    }
                    dp[r] = p * (d - ld.y);
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const frag<T> p = to_operand<T>(s, t), ds = to_operand<T>(dp, t);
#pragma unroll
                    for (int d = 0; d < DIM / 32; ++d) dvacc[d] = mfma(Tile::columns(dt, 32 * n, d, t), p, dvacc[d]);
#pragma unroll
                    for (int d = 0; d < DIM / 32; ++d) dkacc[d] = mfma(Tile::columns(qt, 32 * n, d, t), ds, dkacc[d]);
                }
            }
        }
    }
    if (j < (int)a.k_len) {
        if (mine >= ql) {
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d) dkacc[d] = dvacc[d] = 0.0f;
        }
        store_row(dk + b * a.dk.batch + (uint64_t)j * a.dk.row + kv * a.dk.head, dkacc, a.scale, a.head_dim);
        store_row(dv + b * a.dv.batch + (uint64_t)j * a.dv.row + kv * a.dv.head, dvacc, 1.0f, a.head_dim);
    }
}

struct BackwardPointers { const void *q, *k, *v, *o, *d_o; const float* lse; void *dq, *dk, *dv; float* rows_d; };

template <typename T, int DIM, bool DROP>
static void launch_backward(const AttentionArgs& a, const BackwardPointers& p, hipStream_t s) {
    if (a.q_len) {
        const uint32_t blocks = (a.q_len + BWD_ROWS - 1) / BWD_ROWS;
        hipLaunchKernelGGL((attention_backward_queries_kernel<T, DIM, DROP>), dim3(blocks * a.batch * a.heads), dim3(BWD_THREADS), 0, s, a, (const T*)p.q,
                           (const T*)p.k, (const T*)p.v, (const T*)p.o, p.lse, (const T*)p.d_o, (T*)p.dq, p.rows_d, blocks);
    }
    if (a.k_len) {
        const uint32_t blocks = (a.k_len + BWD_ROWS - 1) / BWD_ROWS;
        timing_before(s);
        hipLaunchKernelGGL((attention_backward_keys_kernel<T, DIM, DROP>), dim3(blocks * a.batch * a.kv_heads), dim3(BWD_THREADS), 0, s, a, (const T*)p.q,
                           (const T*)p.k, (const T*)p.v, p.lse, (const T*)p.d_o, (const float*)p.rows_d, (T*)p.dk, (T*)p.dv, blocks);
        timing_after(s);
    }
}

template <typename T>
static void launch_backward_shape(const AttentionArgs& a, const BackwardPointers& p, hipStream_t s) {
    const bool drop = a.drop.bar != 65536u;
    if (a.head_dim <= 64) drop ? launch_backward<T, 64, true>(a, p, s) : launch_backward<T, 64, false>(a, p, s);
    else drop ? launch_backward<T, 128, true>(a, p, s) : launch_backward<T, 128, false>(a, p, s);
}

}  // namespace okt

extern "C" int okt_attention_backward(const okt_attention* op, const void* d_q, const void* d_k, const void* d_v,
                                      const void* d_o, const float* d_lse, const void* d_do, void* d_dq_out, void* d_dk_out,
                                      void* d_dv_out, void* d_ws, size_t ws_bytes, void* stream) {
    using namespace okt;
    AttentionArgs a;
    if (!attention_args(op, true, a)) return OKT_ERR_INVALID_ARG;
    if (a.batch == 0) return OKT_OK;
    if (a.q_len && (!d_q || !d_o || !d_lse || !d_do || !d_dq_out)) return OKT_ERR_INVALID_ARG;
    if (a.k_len && (!d_k || !d_v || !d_dk_out || !d_dv_out)) return OKT_ERR_INVALID_ARG;
    for (const void* p : {d_q, d_k, d_v, d_o, d_do, (const void*)d_dq_out, (const void*)d_dk_out, (const void*)d_dv_out})
        if (!aligned(p, 16)) return OKT_ERR_INVALID_ARG;
    if (!aligned(d_lse, 4)) return OKT_ERR_INVALID_ARG;
    if (!d_ws || !aligned(d_ws, 256) || ws_bytes < attention_ws_bytes(a.batch, a.heads, a.q_len)) return OKT_ERR_WORKSPACE;
    const BackwardPointers p = {d_q, d_k, d_v, d_o, d_do, d_lse, d_dq_out, d_dk_out, d_dv_out, (float*)d_ws};
    const hipStream_t s = (hipStream_t)stream;
    if (op->dtype == OKT_BF16) launch_backward_shape<__bf16>(a, p, s);
    else launch_backward_shape<_Float16>(a, p, s);
    return launch_status();
}
