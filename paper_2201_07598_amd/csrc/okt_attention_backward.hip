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
//
// With dropout, scaled by c = 65536 / bar where kept:  ds = p (c kept(dp) - D) = c p (kept(dp) - D / c)
// and dv = c sum kept(p) do, so c is applied once at the end, not to every pair.
//
// p and ds are rounded for the second products as in the forward pass; D comes from o as it was stored, whose rounding is
// small beside dP wherever more than a few keys share a row (a row of at most 32 takes it from what it has in registers).
//
// Of 64 columns the vector units are the busiest part (queries 47 %, keys 38 % of all cycles in a padded batch with dropout,
// 34 and 26 without, the matrix units 17 to 21), and no unit is a bound: CUs are empty for a fifth to a quarter of
// the time, and the keys' kernel has 1.8 waves a SIMD to hide its chain.  Of 128 the queries' is bound by the matrix
// units (63 % of a busy CU's time), and the keys', whose sums and operands take more than half of the registers, runs one
// wave a SIMD and waits on its own chain (36 %).  From call to call:
//   32 x 16 heads x 512 x 64, lengths up to 512, bf16, p = 0.1  138-149 us (queries 61, keys 80)
//   2 x 16 heads (4 key heads) x 4096 x 128, causal, bf16       515-535 us, 650 TFLOP/s of visible pairs (200, 360 in a trace)
//   3 x 6 heads (2 key heads) x 197 x 333 x 40, fp16, causal    21-24 us: three dependent launches, 12.6 us of the host
#include "okt_attention.h"

namespace okt {

constexpr int BWD_THREADS = 256;
constexpr int BWD_QUERIES = ATTENTION_QUERIES, BWD_KEYS = ATTENTION_KEYS;
static_assert(BWD_QUERIES == BWD_THREADS / WAVE * 32, "a wave owns 32 queries");

// What the keys' kernel has to know of a query: its log-sum-exp to base 2 (+inf for a row that
// sees nothing, whose probabilities come out as 0), less what that kernel raises probabilities by, and D / c by as much lower.
typedef float2 RowNumbers;

template <typename T, int DIM, bool DROP, bool FINE>
__global__ __launch_bounds__(BWD_THREADS, 2) void attention_backward_queries_kernel(
    AttentionArgs a, const T* q, const T* k, const T* v, const T* o, const float* lse, const T* d_o, T* dq, RowNumbers* rows,
    Places all, uint32_t parts, Divider by_part, float* partial) {
    using Tile = RowTile<T, DIM, BWD_KEYS, BWD_THREADS>;
    __shared__ __attribute__((aligned(1024))) char shared[4 * Tile::BYTES];
    const Place at = place_of(blockIdx.x, all);
    const uint32_t block = quotient(at.block, by_part), part = at.block - block * parts, blocks = quotient(all.blocks, by_part);
    const uint32_t b = quotient(at.unit, a.by_kv), kv = at.unit - b * a.kv_heads, h = kv * a.group + at.head, plane = b * a.heads + h;
    const uint32_t wave = uniform(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const int ql = sequence_length(a.q_lens, b, a.q_len), kl = sequence_length(a.k_lens, b, a.k_len);
    const int q0 = (blocks - 1 - block) * BWD_QUERIES, w0 = q0 + 32 * (int)wave, i = w0 + (int)row_of_lane();
    const int past = kl - ql + 1;
    const auto seen = [&](int query) { const int n = query + past; return query >= ql ? 0 : !a.causal || n > kl ? kl : n < 0 ? 0 : n; };
    const int keys = q0 < ql ? seen(q0 + BWD_QUERIES < ql ? q0 + BWD_QUERIES - 1 : ql - 1) : 0;
    // a lane past the last query goes along as that one, so that no tile is masked for its sake
    const int mine = q0 < ql ? seen(i < ql ? i : ql - 1) : 0, wave_least = w0 < ql ? seen(w0) : 0;
    const int wave_most = w0 < ql ? seen(w0 + 32 < ql ? w0 + 31 : ql - 1) : 0;
    const float drop_scale = DROP ? a.drop.scale : 1.0f;
    // the tiles of this part; part 0 also leaves the rows' numbers
    const Part mine_of = part_of((keys + BWD_KEYS - 1) / BWD_KEYS, part, by_part);
    const int begin = mine_of.first * BWD_KEYS, end = mine_of.last * BWD_KEYS < keys ? mine_of.last * BWD_KEYS : keys;

    f32x16 acc[DIM / 32];
    float base = INFINITY, sum = 0.0f;            // log-sum-exp, D / c
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) acc[d] = 0.0f;
    if (begin < end) {
        const T* kb = k + b * a.k.batch + kv * a.k.head;
        const T* vb = v + b * a.v.batch + kv * a.v.head;
        const uint64_t row = i < ql ? i : ql - 1;
        const T* q_row = q + b * a.q.batch + row * a.q.row + h * a.q.head;
        const T* do_row = d_o + b * a.d_o.batch + row * a.d_o.row + h * a.d_o.head;
        const T* o_row = o + b * a.o.batch + row * a.o.row + h * a.o.head;
        const uint32_t k_row = (uint32_t)a.k.row * 2, v_row = (uint32_t)a.v.row * 2;
        const typename Tile::Places k_at(k_row, a.head_dim), v_at(v_row, a.head_dim);
        const uint32_t lds = lds_address(shared);
        typename Tile::Stream k_tiles(kb, k_row, begin, kl, a.head_dim), v_tiles(vb, v_row, begin, kl, a.head_dim);
        k_tiles.fetch(lds, k_at);
        v_tiles.fetch(lds + Tile::BYTES, v_at);
        frag<T> qf[DIM / 16], df[DIM / 16];
        row_operands<DIM>(qf, q_row, a.head_dim);
        row_operands<DIM>(df, do_row, a.head_dim);
        frag<T> of[DIM / 16];
        row_operands<DIM>(of, o_row, a.head_dim);
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            const f32x8 x = __builtin_convertvector(df[s], f32x8), y = __builtin_convertvector(of[s], f32x8);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum = __builtin_fmaf(x[e], y[e], sum);
        }
        sum = mine > 0 && drop_scale > 0.0f ? sum_halves(sum) / drop_scale : 0.0f;      // all dropped: no gradient anyway
        if (mine > 0) base = lse[(uint64_t)plane * a.q_len + row] * 1.44269504088896f;
        const TileReads reads = Tile::reads();
        RandomKey key = {0, 0};
        if (DROP) key = random_key(a.seed);

        for (int key0 = begin, turn = 0; key0 < end; key0 += BWD_KEYS, turn ^= 1) {
            fetched();
            const char* kt = shared + turn * 2 * Tile::BYTES;
            const char* vt = kt + Tile::BYTES;
            if (key0 + BWD_KEYS < end) {
                const uint32_t next = lds + (turn ^ 1) * 2 * Tile::BYTES;
                k_tiles.fetch(next, k_at);
                v_tiles.fetch(next + Tile::BYTES, v_at);
            }
            if (key0 >= wave_most) continue;
            const bool masked = key0 + BWD_KEYS > wave_least;
#pragma unroll
            for (int n = 0; n < BWD_KEYS / 32; ++n) {
                f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) {
                    s = mfma(Tile::rows(kt, reads, 32 * n, e), qf[e], s);
                    dp = mfma(Tile::rows(vt, reads, 32 * n, e), df[e], dp);
                }
                if (DROP) {
                    uint32_t w[8];
                    kept_keys(w, i, key0 + 32 * n, plane, key, a.site);
#pragma unroll
                    for (int r = 0; r < 16; ++r) dp[r] = kept_element(w, r, a.drop.bar) ? dp[r] : 0.0f;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -base));
                if (masked) {
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[r] = key0 + 32 * n + 16 * (int)(lane / 32) + r < mine ? s[r] : 0.0f;
                }
                if (n == 0 && key0 == 0) {
                    // A row that sees no key past this tile takes D from what it has here, sum_j p dP: few
                    // probabilities are large ones, and the rounding of o would show in dP - D.  Taken
                    // from the largest dP on, so that a row with one key gets its dP itself and ds = 0.
                    float from = -INFINITY, few = 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) from = fmaxf(from, 16 * (int)(lane / 32) + r < mine ? dp[r] : -INFINITY);
                    from = mine > 0 ? max_halves(from) : 0.0f;
#pragma unroll
                    for (int r = 0; r < 16; ++r) few = __builtin_fmaf(s[r], dp[r] - from, few);
                    few = from + sum_halves(few);
                    sum = mine > 0 && mine <= 32 ? few : sum;
                }
#pragma unroll
                for (int r = 0; r < 16; ++r) s[r] *= dp[r] - sum;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const Operand<T, FINE> ds(s, t);
#pragma unroll
                    for (int d = 0; d < DIM / 32; ++d) acc[d] = mfma(Tile::columns(kt, reads, 32 * n, d, t), ds, acc[d]);
                }
            }
        }
    }
    if (part == 0 && lane < 32 && i < ql)
        rows[(uint64_t)plane * a.q_len + i] = make_float2(base - Raised<T>::keys, sum / Raised<T>::keys_factor);
    if (i < (int)a.q_len) {
        T* out = dq + b * a.dq.batch + (uint64_t)i * a.dq.row + h * a.dq.head;
        if (mine == 0 || i >= ql) {
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d) acc[d] = 0.0f;
        }
        if (parts > 1) store_partial(partial + (((uint64_t)part * a.batch * a.heads + plane) * a.q_len + i) * DIM, acc, a.scale * drop_scale);
        else store_row(out, acc, a.scale * drop_scale, a.head_dim);
    }
}

template <typename T, int DIM, bool DROP, bool FINE>
__global__ __launch_bounds__(BWD_THREADS, DIM == 64 ? 2 : 1) void attention_backward_keys_kernel(
    AttentionArgs a, const T* q, const T* k, const T* v, const T* d_o, const RowNumbers* rows, T* dk, T* dv, Places all,
    uint32_t parts, Divider by_part, float* partial) {
    using Shape = KeysShape<DIM>;
    constexpr int TILE = Shape::TILE, EACH = 32 * Shape::HALVES;           // queries of a tile, from a wave's 32 to its next
    using Tile = RowTile<T, DIM, TILE, BWD_THREADS>;
    constexpr int NUMBERS = TILE * (int)sizeof(RowNumbers) < 1024 ? 1024 : TILE * (int)sizeof(RowNumbers);
    constexpr int BUFFER = 2 * Tile::BYTES + NUMBERS;
    constexpr float LOWER = 1.0f / Raised<T>::keys_factor;      // p comes raised, so that ds = p (kept(dp) - D / c) takes the rest lowered
    __shared__ __attribute__((aligned(1024))) char shared[2 * BUFFER];
    const Place at = place_of(blockIdx.x, all);
    const uint32_t block = quotient(at.block, by_part), share = at.block - block * parts;
    const uint32_t b = quotient(at.unit, a.by_kv), kv = at.unit - b * a.kv_heads;
    const uint32_t wave = uniform(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const uint32_t part = wave / Shape::GROUPS;
    const int ql = sequence_length(a.q_lens, b, a.q_len), kl = sequence_length(a.k_lens, b, a.k_len);
    const int k0 = block * (Shape::GROUPS * 32), w0 = k0 + 32 * (int)(wave % Shape::GROUPS), j = w0 + (int)row_of_lane();
    // the first query that sees a key: any key, the workgroup's, the wave's first and last, the lane's
    const auto first_for = [&](int key) { const int n = a.causal ? key - (kl - ql) : 0; return n < 0 ? 0 : n; };
    const int lo = first_for(0), begin = first_for(k0) / TILE * TILE;
    // a lane past the last key goes along as that one, so that no tile is masked for its sake; queries past
    // the last need no mask, since their rows arrive as zeros
    const int mine = k0 < kl ? first_for(j < kl ? j : kl - 1) : ql;
    const int wave_least = w0 < kl ? first_for(w0) : ql + TILE, wave_most = first_for(w0 + 31 < kl ? w0 + 31 : kl - 1);
    const int tiles = k0 < kl && begin < ql ? (ql - begin + TILE - 1) / TILE : 0;
    const float drop_scale = DROP ? a.drop.scale : 1.0f;
    // the steps of this share: the tiles of every head of the group, head after head
    const Part steps = part_of(tiles * (int)a.group, share, by_part);

    f32x16 dkacc[DIM / 32], dvacc[DIM / 32];
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) dkacc[d] = dvacc[d] = 0.0f;
    if (steps.first < steps.last) {
        const uint32_t q_row = (uint32_t)a.q.row * 2, do_row = (uint32_t)a.d_o.row * 2, lds = lds_address(shared);
        const typename Tile::Places q_at(q_row, a.head_dim), do_at(do_row, a.head_dim);
        // the tile that is fetched next, head after head of the group
        uint32_t fetch_head = kv * a.group + steps.first / tiles;
        int fetch_query = begin + steps.first % tiles * TILE;
        const auto q_of = [&](int first) { return typename Tile::Stream(q + b * a.q.batch + fetch_head * a.q.head, q_row, first, ql, a.head_dim); };
        const auto do_of = [&](int first) { return typename Tile::Stream(d_o + b * a.d_o.batch + fetch_head * a.d_o.head, do_row, first, ql, a.head_dim); };
        typename Tile::Stream q_tiles = q_of(fetch_query), do_tiles = do_of(fetch_query);
        const auto fetch = [&](int turn) {
            const uint32_t to = lds + turn * BUFFER;
            q_tiles.fetch(to, q_at, lo - fetch_query);
            do_tiles.fetch(to + Tile::BYTES, do_at, lo - fetch_query);
            const RowNumbers* from = rows + ((uint64_t)b * a.heads + fetch_head) * a.q_len;
            if (wave == 0) fetch_line(to + 2 * Tile::BYTES, from + fetch_query, from + ql);
            fetch_query += TILE;
            if (fetch_query >= ql) {
                fetch_query = begin;
                ++fetch_head;
                q_tiles = q_of(begin);
                do_tiles = do_of(begin);
            }
        };
        fetch(0);
        const uint64_t row = j < kl ? j : kl - 1;
        const T* k_row = k + b * a.k.batch + row * a.k.row + kv * a.k.head;
        const T* v_row = v + b * a.v.batch + row * a.v.row + kv * a.v.head;
        frag<T> kf[DIM / 16], vf[DIM / 16];
        row_operands<DIM>(kf, k_row, a.head_dim);
        row_operands<DIM>(vf, v_row, a.head_dim);
        const TileReads reads = Tile::reads();
        RandomKey key = {0, 0};
        if (DROP) key = random_key(a.seed);
        uint32_t plane = b * a.heads + kv * a.group + steps.first / tiles;
        int query0 = begin + steps.first % tiles * TILE;
        for (int it = steps.first, turn = 0; it < steps.last; ++it, turn ^= 1) {
            fetched();
            const char* qt = shared + turn * BUFFER;
            const char* dt = qt + Tile::BYTES;
            const RowNumbers* numbers = reinterpret_cast<const RowNumbers*>(dt + Tile::BYTES);
            if (it + 1 < steps.last) fetch(turn ^ 1);
            // a wave's part of a tile are every HALVES-th 32 queries, so that the parts of a short sequence are
            // alike (6 heads of 50 x 50 x 128: 24.4 us with a half of the tile each, so 21.1)
            const int own0 = query0 + 32 * (int)part;
            if (own0 + TILE - EACH + 32 > wave_least && own0 < ql) {
                const bool masked = own0 < wave_most;
#pragma unroll 1
                for (int n = 0; n < TILE / EACH; ++n) {
                    if (Shape::HALVES == 2 && own0 + EACH * n >= ql) break;
                    const uint32_t slot0 = 32 * part + EACH * n;
                    f32x16 s = 0.0f, dp = 0.0f;
#pragma unroll
                    for (int e = 0; e < DIM / 16; ++e) {
                        s = mfma(Tile::rows(qt, reads, slot0, e), kf[e], s);
                        dp = mfma(Tile::rows(dt, reads, slot0, e), vf[e], dp);
                    }
                    const float4* number = reinterpret_cast<const float4*>(numbers + slot0 + 16 * (lane / 32));
                    float few[16];
#pragma unroll
                    for (int r = 0; r < 16; r += 2) {
                        const float4 two = number[r / 2];
                        s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a.scale_log2, -two.x));
                        s[r + 1] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r + 1], a.scale_log2, -two.z));
                        few[r] = two.y;
                        few[r + 1] = two.w;
                    }
                    if (masked) {
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int i = own0 + EACH * n + 16 * (int)(lane / 32) + r;
                            s[r] = i >= mine ? s[r] : 0.0f;
                        }
                    }
                    if (DROP) {
                        uint32_t w[8];
                        kept_queries(w, j, own0 + EACH * n, plane, key, a.site);
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const bool keep = kept_element(w, r, a.drop.bar);
                            const float p = s[r];
                            s[r] = keep ? p : 0.0f;
                            dp[r] = p * __builtin_fmaf(keep ? dp[r] : 0.0f, LOWER, -few[r]);
                        }
                    } else {
#pragma unroll
                        for (int r = 0; r < 16; ++r) dp[r] = s[r] * __builtin_fmaf(dp[r], LOWER, -few[r]);
                    }
#pragma unroll
                    for (int t = 0; t < 2; ++t) {
                        const Operand<T, FINE> p(s, t), ds(dp, t);
#pragma unroll
                        for (int d = 0; d < DIM / 32; ++d) {
                            dvacc[d] = mfma(Tile::columns(dt, reads, slot0, d, t), p, dvacc[d]);
                            dkacc[d] = mfma(Tile::columns(qt, reads, slot0, d, t), ds, dkacc[d]);
                        }
                    }
                }
            }
            query0 += TILE;
            if (query0 >= ql) {
                query0 = begin;
                ++plane;
            }
        }
        if (Shape::HALVES == 2) {                              // the waves of the other part hand over their sums
            f32x16* sums = reinterpret_cast<f32x16*>(shared) + (wave % Shape::GROUPS) * (DIM / 16) * WAVE + lane;
            __syncthreads();
            if (part == 1) {
#pragma unroll
                for (int d = 0; d < DIM / 32; ++d) {
                    sums[2 * d * WAVE] = dkacc[d];
                    sums[(2 * d + 1) * WAVE] = dvacc[d];
                }
            }
            __syncthreads();
            if (part == 0) {
#pragma unroll
                for (int d = 0; d < DIM / 32; ++d) {
                    dkacc[d] += sums[2 * d * WAVE];
                    dvacc[d] += sums[(2 * d + 1) * WAVE];
                }
            }
        }
    }
    if (part == 0 && j < (int)a.k_len) {
        if (mine >= ql || j >= kl) {
#pragma unroll
            for (int d = 0; d < DIM / 32; ++d) dkacc[d] = dvacc[d] = 0.0f;
        }
        if (parts > 1) {
            float* to = partial + (((uint64_t)share * a.batch * a.kv_heads + b * a.kv_heads + kv) * a.k_len + j) * DIM;
            store_partial(to, dkacc, a.scale * drop_scale);
            store_partial(to + (uint64_t)parts * a.batch * a.kv_heads * a.k_len * DIM, dvacc, drop_scale * LOWER);
            return;
        }
        store_row(dk + b * a.dk.batch + (uint64_t)j * a.dk.row + kv * a.dk.head, dkacc, a.scale * drop_scale, a.head_dim);
        store_row(dv + b * a.dv.batch + (uint64_t)j * a.dv.row + kv * a.dv.head, dvacc, drop_scale * LOWER, a.head_dim);
    }
}

// Adds the parts of up to three tensors, four columns a lane, always in the same order.
struct Sum { const float* from; void* to; Strides strides; uint64_t rows; uint32_t parts, length, heads; };
struct Sums { Sum of[3]; };

template <typename T, int DIM>
__global__ __launch_bounds__(BWD_THREADS) void attention_add_kernel(Sums sums, uint32_t head_dim) {
    typedef T four __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const Sum& s = sums.of[blockIdx.y];
    const uint64_t at = (uint64_t)blockIdx.x * BWD_THREADS + threadIdx.x, row = at / (DIM / 4);
    const uint32_t d = at % (DIM / 4) * 4;
    if (row >= s.rows || d >= head_dim) return;
    f32x4 sum = 0.0f;
#pragma unroll 4
    for (uint32_t p = 0; p < s.parts; ++p) sum += *reinterpret_cast<const f32x4*>(s.from + (p * s.rows + row) * DIM + d);
    const uint64_t i = row % s.length, plane = row / s.length, h = plane % s.heads, b = plane / s.heads;
    *reinterpret_cast<four*>((T*)s.to + b * s.strides.batch + i * s.strides.row + h * s.strides.head + d) = __builtin_convertvector(sum, four);
}

struct BackwardPointers { const void *q, *k, *v, *o, *d_o; const float* lse; void *dq, *dk, *dv; char* ws; };

template <typename T, int DIM, bool DROP, bool FINE>
static int launch_backward(const AttentionArgs& a, const AttentionPlan& plan, const BackwardPointers& p, hipStream_t s) {
    RowNumbers* rows = (RowNumbers*)(p.ws + plan.rows_at);
    float *dq_sums = (float*)(p.ws + plan.dq_at), *dkv_sums = (float*)(p.ws + plan.dkv_at);
    Sums sums = {};
    uint32_t n = 0;
    if (a.q_len) {
        const uint32_t blocks = (a.q_len + BWD_QUERIES - 1) / BWD_QUERIES, parts = plan.query_parts;
        hipLaunchKernelGGL((attention_backward_queries_kernel<T, DIM, DROP, FINE>), dim3((unsigned)plan.query_groups),
                           dim3(BWD_THREADS), 0, s, a, (const T*)p.q, (const T*)p.k, (const T*)p.v, (const T*)p.o, p.lse,
                           (const T*)p.d_o, (T*)p.dq, rows,
                           places(a.batch * a.kv_heads, a.group, blocks * parts, window_of(a.causal, a.k_len, DIM, a.group)), parts,
                           divider(parts), dq_sums);
        if (const int status = launch_status()) return status;          // the keys' kernel would read what this one has not written
        if (parts > 1) sums.of[n++] = {dq_sums, p.dq, a.dq, (uint64_t)a.batch * a.heads * a.q_len, parts, a.q_len, a.heads};
    }
    if (a.k_len) {
        constexpr uint32_t KEYS = KeysShape<DIM>::GROUPS * 32;
        const uint32_t blocks = (a.k_len + KEYS - 1) / KEYS, parts = plan.key_parts;
        const uint64_t keys = (uint64_t)a.batch * a.kv_heads * a.k_len;
        timing_before(s);
        hipLaunchKernelGGL((attention_backward_keys_kernel<T, DIM, DROP, FINE>), dim3((unsigned)plan.key_groups),
                           dim3(BWD_THREADS), 0, s, a, (const T*)p.q, (const T*)p.k, (const T*)p.v, (const T*)p.d_o,
                           (const RowNumbers*)rows, (T*)p.dk, (T*)p.dv, 
                           places(a.batch * a.kv_heads, 1, blocks * parts, window_of(a.causal, a.q_len, DIM, 1)), parts, divider(parts),
                           dkv_sums);
        timing_after(s);
        if (const int status = launch_status()) return status;
        if (parts > 1) {
            sums.of[n++] = {dkv_sums, p.dk, a.dk, keys, parts, a.k_len, a.kv_heads};
            sums.of[n++] = {dkv_sums + parts * keys * DIM, p.dv, a.dv, keys, parts, a.k_len, a.kv_heads};
        }
    }
    if (n) {
        uint64_t most = 0;
        for (uint32_t i = 0; i < n; ++i) most = sums.of[i].rows > most ? sums.of[i].rows : most;
        hipLaunchKernelGGL((attention_add_kernel<T, DIM>), dim3((unsigned)((most * (DIM / 4) + BWD_THREADS - 1) / BWD_THREADS), n),
                           dim3(BWD_THREADS), 0, s, sums, a.head_dim);
    }
    return launch_status();
}

template <typename T, bool FINE>
static int launch_backward_columns(const AttentionArgs& a, const AttentionPlan& plan, const BackwardPointers& p, hipStream_t s) {
    const bool drop = a.drop.bar != 65536u;
    if (plan.dim == 64) return drop ? launch_backward<T, 64, true, FINE>(a, plan, p, s) : launch_backward<T, 64, false, FINE>(a, plan, p, s);
    return drop ? launch_backward<T, 128, true, FINE>(a, plan, p, s) : launch_backward<T, 128, false, FINE>(a, plan, p, s);
}

template <typename T>
static int launch_backward_shape(const AttentionArgs& a, const AttentionPlan& plan, const BackwardPointers& p, hipStream_t s) {
    return plan.fine ? launch_backward_columns<T, true>(a, plan, p, s) : launch_backward_columns<T, false>(a, plan, p, s);
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
    const AttentionPlan plan = attention_plan(a.batch, a.heads, a.kv_heads, a.q_len, a.k_len, a.head_dim, a.drop.bar != 65536u);
    if (plan.query_groups > LAUNCH_GROUPS || plan.key_groups > LAUNCH_GROUPS) return OKT_ERR_INVALID_ARG;
    if (!d_ws || !aligned(d_ws, 256) || ws_bytes < plan.bytes) return OKT_ERR_WORKSPACE;
    const auto there = [](uint32_t length, const void* p) { return length ? p : nullptr; };
    const void* const tensors[] = {there(a.q_len, d_dq_out), there(a.k_len, d_dk_out), there(a.k_len, d_dv_out), there(a.q_len, d_q),
                                   there(a.k_len, d_k), there(a.k_len, d_v), there(a.q_len, d_o), there(a.q_len, d_do)};
    for (int out = 0; out < 3; ++out)
        for (int other = out + 1; other < 8; ++other)
            if (same_place(tensors[out], tensors[other], a.head_dim)) return OKT_ERR_INVALID_ARG;
    const BackwardPointers p = {d_q, d_k, d_v, d_o, d_do, d_lse, d_dq_out, d_dk_out, d_dv_out, (char*)d_ws};
    const hipStream_t s = (hipStream_t)stream;
    return op->dtype == OKT_BF16 ? launch_backward_shape<__bf16>(a, plan, p, s) : launch_backward_shape<_Float16>(a, plan, p, s);
}
