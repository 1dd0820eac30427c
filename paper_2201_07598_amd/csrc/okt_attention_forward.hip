// okt_attention_forward: one pass over the keys with a running maximum and sum.
//
// A wave owns 32 queries, a workgroup four waves; the keys and values come by in tiles of
// 64 rows that all four share in LDS, the next tile on its way while one is used.  Scores
// are taken transposed (keys down, queries across): a lane then holds one query's
// scores, so maximum and sum stay in the lane but for one exchange with the lane 32 away,
// and the probabilities are the second product's operand as they lie.
//
// With 64 columns or fewer the vector units have more to do than the matrix units: 64 scores take 35 cycles of a SIMD
// there (60 with dropout, as counted) against 16 of their two products.  In a padded batch of short sequences that work
// fills 38 % of all cycles (49 with dropout); a third of the CUs' time they have no workgroup, before the first tiles
// and behind the longest sequences, and the rest is waiting.  From call to call:
//   32 x 16 heads x 512 x 64, lengths up to 512, bf16, p = 0.1  49-56 us (p = 0: 42; the kernels 51 and 35 in a trace)
//   2 x 16 heads (4 key heads) x 4096 x 128, causal, bf16       145-150 us, 940 TFLOP/s of visible pairs (fp16 167)
//   12 heads x 128 x 64                                         8-10 us, most of it the host's; the kernel 6, two tiles
//   one query of 12 heads over 32768 keys of 128                53-58 us, 3.6 TB/s
//   64 x 8 groups of 4 heads of one query, 4096 keys of 128     193 us, 5.6 TB/s
#include "okt_attention.h"

namespace okt {

constexpr int FWD_THREADS = 256;
constexpr int FWD_QUERIES = ATTENTION_QUERIES, FWD_KEYS = ATTENTION_KEYS;
static_assert(FWD_QUERIES == FWD_THREADS / WAVE * 32, "a wave owns 32 queries");

// A running sum of many terms and what its roundings have added too much (Kahan's summation): rows may be
// millions of keys long, and terms that are alike are rounded alike, so that a plain sum of a million of 0.3 is
// 0.6 % off, and lse with it, from which the backward pass takes every probability.  The probabilities of a tile are
// added pairwise first.  Four operations a tile: 16 x 4096 x 4096 x 64 161 -> 163 us, 128 columns causal 148.7 -> 149.6.
struct CompensatedSum {
    float sum, over;
    __device__ __forceinline__ void add(float v) {
        const float term = v - over, next = sum + term;
        over = (next - sum) - term;
        sum = next;
    }
};

__device__ __forceinline__ float sum_sixteen(const f32x16& v) {
    const auto four = [&](int r) { return (v[r] + v[r + 1]) + (v[r + 2] + v[r + 3]); };
    return (four(0) + four(4)) + (four(8) + four(12));
}

// PACKED: few queries, whose rows of all heads of a group are taken one after the other as the
// rows of one block, so that the group's keys come by once and not once a head.
template <typename T, int DIM, bool DROP, bool PACKED, bool FINE>
__global__ __launch_bounds__(FWD_THREADS, 2) void attention_forward_kernel(AttentionArgs a, const T* q, const T* k, const T* v,
                                                                           T* o, float* lse, Places all, uint32_t parts,
                                                                           Divider by_part, Divider by_query,
                                                                           float* partial, float2* sums) {
    static_assert(!(DROP && PACKED), "neighbouring rows of a block share its random numbers");
    using Tile = RowTile<T, DIM, FWD_KEYS, FWD_THREADS>;
    __shared__ __attribute__((aligned(1024))) char shared[4 * Tile::BYTES];
    const Place at = place_of(blockIdx.x, all);
    const uint32_t block = quotient(at.block, by_part), part = at.block - block * parts, blocks = quotient(all.blocks, by_part);
    const uint32_t b = quotient(at.unit, a.by_kv), kv = at.unit - b * a.kv_heads;
    const uint32_t wave = uniform(threadIdx.x / WAVE), lane = threadIdx.x % WAVE;
    const int ql = sequence_length(a.q_lens, b, a.q_len), kl = sequence_length(a.k_lens, b, a.k_len);
    // the block's first row, the wave's, the lane's; which head and query that is
    const int q0 = (blocks - 1 - block) * FWD_QUERIES, w0 = q0 + 32 * (int)wave, row = w0 + (int)row_of_lane();
    const int rows = PACKED ? (int)(a.group * a.q_len) : (int)a.q_len;
    const uint32_t in_group = PACKED ? quotient(row < rows ? row : rows - 1, by_query) : at.head;
    const int i = PACKED ? row - (int)(in_group * a.q_len) : row;           // past the last row past the last query, too
    const uint32_t h = kv * a.group + in_group, plane = b * a.heads + h;

    // keys that a query sees; the most of the workgroup's queries, the least and most of the wave's
    const int past = kl - ql + 1;
    const auto seen = [&](int query) { const int n = query + past; return query >= ql ? 0 : !a.causal || n > kl ? kl : n < 0 ? 0 : n; };
    const int last = ql - 1, there = PACKED ? (ql ? rows : 0) : ql;         // rows that have a query
    const int keys = q0 >= there ? 0 : seen(PACKED || q0 + FWD_QUERIES >= ql ? last : q0 + FWD_QUERIES - 1);
    // a lane past the last query goes along as that one, so that no tile is masked for its sake
    const int mine = q0 < there ? seen(i < ql ? i : last) : 0;
    const int wave_least = w0 < there ? seen(PACKED ? 0 : w0) : 0, wave_most = w0 < there ? seen(PACKED || w0 + 32 >= ql ? last : w0 + 31) : 0;

    // the tiles of this part
    const Part mine_of = part_of((keys + FWD_KEYS - 1) / FWD_KEYS, part, by_part);
    const int begin = mine_of.first * FWD_KEYS, end = mine_of.last * FWD_KEYS < keys ? mine_of.last * FWD_KEYS : keys;

    f32x16 acc[DIM / 32];
    float top = -INFINITY;                        // of the scores times scale_log2, less what probabilities are raised by
    CompensatedSum total = {0.0f, 0.0f};
#pragma unroll
    for (int d = 0; d < DIM / 32; ++d) acc[d] = 0.0f;
    if (begin < end) {
        const T* kb = k + b * a.k.batch + kv * a.k.head;
        const T* vb = v + b * a.v.batch + kv * a.v.head;
        const uint32_t k_row = (uint32_t)a.k.row * 2, v_row = (uint32_t)a.v.row * 2;
        const typename Tile::Places k_at(k_row, a.head_dim), v_at(v_row, a.head_dim);
        const uint32_t lds = lds_address(shared);
        typename Tile::Stream k_tiles(kb, k_row, begin, kl, a.head_dim), v_tiles(vb, v_row, begin, kl, a.head_dim);
        k_tiles.fetch(lds, k_at);
        v_tiles.fetch(lds + Tile::BYTES, v_at);
        const T* qrow = q + b * a.q.batch + (uint64_t)(i < ql ? i : last) * a.q.row + h * a.q.head;
        frag<T> qf[DIM / 16];
        row_operands<DIM>(qf, qrow, a.head_dim);
        const TileReads reads = Tile::reads();
        RandomKey key = {0, 0};
        if (DROP) key = random_key(a.seed);
        for (int key0 = begin, turn = 0; key0 < end; key0 += FWD_KEYS, turn ^= 1) {
            fetched();
            const char* kt = shared + turn * 2 * Tile::BYTES;
            const char* vt = kt + Tile::BYTES;
            if (key0 + FWD_KEYS < end) {
                const uint32_t next = lds + (turn ^ 1) * 2 * Tile::BYTES;
                k_tiles.fetch(next, k_at);
                v_tiles.fetch(next + Tile::BYTES, v_at);
            }
            if (key0 >= wave_most) continue;
            f32x16 s[FWD_KEYS / 32];
#pragma unroll
            for (int n = 0; n < FWD_KEYS / 32; ++n) {
                s[n] = 0.0f;
#pragma unroll
                for (int e = 0; e < DIM / 16; ++e) s[n] = mfma(Tile::rows(kt, reads, 32 * n, e), qf[e], s[n]);
            }
            if (key0 + FWD_KEYS > wave_least) {                // some of the tile is hidden from some lane
#pragma unroll
                for (int n = 0; n < FWD_KEYS / 32; ++n)
#pragma unroll
                    for (int r = 0; r < 16; ++r)
                        s[n][r] = key0 + 32 * n + 16 * (int)(lane / 32) + r < mine ? s[n][r] : -INFINITY;
            }
            float most = s[0][0];
#pragma unroll
            for (int n = 0; n < FWD_KEYS / 32; ++n)
#pragma unroll
                for (int r = 0; r < 16; ++r) most = fmaxf(most, s[n][r]);
            most = __builtin_fmaf(max_halves(most), a.scale_log2, -Raised<T>::forward);
            // Sums are kept relative to `top`, which follows the maximum in steps: as long as no
            // lane's has grown by more than a factor of 2^8, which changes neither the relative precision of
            // a probability nor of a sum, there is nothing to rescale.
            if (__any(most > top + 8.0f)) {
                most = fmaxf(top, most);
                const float fade = __builtin_amdgcn_exp2f(top - (most == -INFINITY ? 0.0f : most));
                top = most;
                total.sum *= fade;
                total.over *= fade;
#pragma unroll
                for (int d = 0; d < DIM / 32; ++d) acc[d] *= fade;
            }
            const float base = top == -INFINITY ? 0.0f : top;
            float of_tile[FWD_KEYS / 32];
#pragma unroll
            for (int n = 0; n < FWD_KEYS / 32; ++n) {
#pragma unroll
                for (int r = 0; r < 16; ++r) s[n][r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[n][r], a.scale_log2, -base));
                of_tile[n] = sum_sixteen(s[n]);
                if (DROP) {
                    uint32_t w[8];
                    kept_keys(w, i, key0 + 32 * n, plane, key, a.site);
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[n][r] = kept_element(w, r, a.drop.bar) ? s[n][r] : 0.0f;
                }
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    const Operand<T, FINE> p(s[n], t);
#pragma unroll
                    for (int d = 0; d < DIM / 32; ++d) acc[d] = mfma(Tile::columns(vt, reads, 32 * n, d, t), p, acc[d]);
                }
            }
            total.add(of_tile[0] + of_tile[1]);
        }
    }
    const float sum = sum_halves(total.sum - total.over);
    if (row >= rows) return;
    if (parts > 1) {
        const uint64_t to = ((uint64_t)part * a.batch * a.heads + plane) * a.q_len + i;
        store_partial(partial + to * DIM, acc, 1.0f);
        if (lane < 32) sums[to] = make_float2(i < ql ? top : -INFINITY, sum);
        return;
    }
    store_row(o + b * a.o.batch + (uint64_t)i * a.o.row + h * a.o.head, acc, mine > 0 && i < ql ? a.drop.scale / sum : 0.0f, a.head_dim);
    if (lse && lane < 32)
        lse[(uint64_t)plane * a.q_len + i] = mine > 0 && i < ql ? (top + __builtin_amdgcn_logf(sum)) * 0.693147180559945f : -INFINITY;
}

// Joins the parts of a row: o = sum 2^(top - most) acc / sum 2^(top - most) total.  DIM / 4 lanes a
// row, four columns a lane.
template <typename T, int DIM>
__global__ __launch_bounds__(FWD_THREADS) void attention_join_kernel(AttentionArgs a, T* o, float* lse, uint32_t parts,
                                                                     const float* partial, const float2* sums) {
    constexpr uint32_t LANES = DIM / 4, AT_ONCE = 8;
    typedef T four __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const uint64_t rows = (uint64_t)a.batch * a.heads * a.q_len;
    const uint64_t row = (uint64_t)blockIdx.x * (FWD_THREADS / LANES) + threadIdx.x / LANES;
    const uint32_t d = threadIdx.x % LANES * 4;
    if (row >= rows) return;
    float most = -INFINITY, total = 0.0f;
    f32x4 acc = 0.0f;
    for (uint32_t p0 = 0; p0 < parts; p0 += AT_ONCE) {          // that many parts' loads are on their way together
        float2 part[AT_ONCE];
        f32x4 v[AT_ONCE];
        float top = most;
#pragma unroll
        for (uint32_t n = 0; n < AT_ONCE; ++n) {
            const uint64_t at = (p0 + n < parts ? p0 + n : parts - 1) * rows + row;
            part[n] = sums[at];
            v[n] = *reinterpret_cast<const f32x4*>(partial + at * DIM + d);
            if (p0 + n >= parts) part[n].x = -INFINITY;
            top = fmaxf(top, part[n].x);
        }
        const float fade = most == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(most - top);
        most = top;
        acc *= fade;
        total *= fade;
#pragma unroll
        for (uint32_t n = 0; n < AT_ONCE; ++n) {
            const float weight = part[n].x == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(part[n].x - most);
            total = __builtin_fmaf(part[n].y, weight, total);
            acc += weight * v[n];
        }
    }
    const bool any = most != -INFINITY;
    acc *= any ? a.drop.scale / total : 0.0f;
    const uint32_t i = row % a.q_len, h = row / a.q_len % a.heads, b = row / a.q_len / a.heads;
    if (d < a.head_dim)
        *reinterpret_cast<four*>(o + b * a.o.batch + (uint64_t)i * a.o.row + h * a.o.head + d) = __builtin_convertvector(acc, four);
    if (lse && d == 0) lse[row] = any ? (most + __builtin_amdgcn_logf(total)) * 0.693147180559945f : -INFINITY;
}

template <typename T, int DIM, bool FINE>
static int launch_forward(const AttentionArgs& a, const AttentionPlan& plan, const void* q, const void* k, const void* v, void* o,
                           float* lse, void* ws, hipStream_t s) {
    const uint64_t rows = (uint64_t)a.batch * a.heads * a.q_len;
    const uint32_t block_rows = plan.packed ? a.group * a.q_len : a.q_len, block_heads = plan.packed ? 1 : a.group;
    const uint32_t blocks = (block_rows + FWD_QUERIES - 1) / FWD_QUERIES, parts = plan.forward_parts;
    float* partial = (float*)ws;
    float2* sums = (float2*)(partial + parts * rows * DIM);
    auto* kernel = a.drop.bar != 65536u ? attention_forward_kernel<T, DIM, true, false, FINE>
                   : plan.packed        ? attention_forward_kernel<T, DIM, false, true, FINE>
                                        : attention_forward_kernel<T, DIM, false, false, FINE>;
    timing_before(s);
    hipLaunchKernelGGL(kernel, dim3((unsigned)plan.forward_groups), dim3(FWD_THREADS), 0, s, a, (const T*)q,
                       (const T*)k, (const T*)v, (T*)o, lse,
                       places(a.batch * a.kv_heads, block_heads, blocks * parts, window_of(a.causal && !plan.packed, a.k_len, DIM, a.group)),
                       parts, divider(parts), divider(a.q_len), partial, sums);
    timing_after(s);
    int status = launch_status();
    if (status == OKT_OK && parts > 1) {
        hipLaunchKernelGGL((attention_join_kernel<T, DIM>), dim3((unsigned)((rows * (DIM / 4) + FWD_THREADS - 1) / FWD_THREADS)),
                           dim3(FWD_THREADS), 0, s, a, (T*)o, lse, parts, (const float*)partial, (const float2*)sums);
        status = launch_status();
    }
    return status;
}

template <typename T>
static int launch_forward_shape(const AttentionArgs& a, const AttentionPlan& plan, const void* q, const void* k, const void* v, void* o,
                                float* lse, void* ws, hipStream_t s) {
    auto* launch = plan.dim == 64 ? (plan.fine ? launch_forward<T, 64, true> : launch_forward<T, 64, false>)
                                  : (plan.fine ? launch_forward<T, 128, true> : launch_forward<T, 128, false>);
    return launch(a, plan, q, k, v, o, lse, ws, s);
}

// Up to so many pairs the second products are taken from p and ds in two parts.  An output of few pairs has its error
// from few roundings: in one part, the error against 64 bits of 2 to 50 queries and keys was up to 2.0 times that of
// outputs rounded once (2 % of 500 drawn sizes over 1.5 times), and from 2^16 pairs on 1.4 to 1.49 times (of 1,280 drawn sizes).  In two parts
// everywhere it would be 1.0 to 1.1 times, and 32 x 16 x 512 x 64 56 -> 67 us, 2 x 16 x 4096 x 128 148 -> 204, their
// gradients 145 -> 174 and 533 -> 678.  Below the bound it costs up to 1 us (2 x 2 x 128 x 128 x 64 gradient 19 -> 20.5).
constexpr uint64_t FINE_PAIRS = 1ull << 16;

AttentionPlan attention_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t q_len, uint32_t k_len, uint32_t head_dim,
                             bool drop) {
    AttentionPlan p;
    p.dim = head_dim <= 64 ? 64 : 128;
    const uint32_t key_block = p.dim == 64 ? KeysShape<64>::GROUPS * 32 : KeysShape<128>::GROUPS * 32;
    const uint32_t query_tile = p.dim == 64 ? KeysShape<64>::TILE : KeysShape<128>::TILE;
    const uint64_t units = (uint64_t)batch * kv_heads, planes = (uint64_t)batch * heads, group = kv_heads ? heads / kv_heads : 0;
    const uint64_t query_blocks = (q_len + ATTENTION_QUERIES - 1) / ATTENTION_QUERIES * planes;
    const uint64_t key_steps = (k_len + ATTENTION_KEYS - 1) / ATTENTION_KEYS;
    const uint64_t rows = planes * q_len, keys = units * k_len;
    const uint64_t query_steps = (q_len + query_tile - 1) / query_tile * group, row_bytes = p.dim * sizeof(float);
    // What a step takes: 0.77, 1.09 and 1.34 us of 64 columns and twice that of 128 (forward, queries, keys).  Where a few
    // workgroups run alone it is 0.7, 0.9 and 1.4 us, and 1.0, 1.4 and 2.0 of 128 columns; with one on every CU, which share
    // the memory, 1.1, 1.4 and 2.0, and 2.1, 2.3 and 6.
    const auto worth = [&](uint64_t workgroups, uint64_t steps, uint64_t step_ns, uint64_t bytes, bool added) {
        return parts_worth(parts_for(workgroups, steps, 1), steps, step_ns * p.dim, 2 * bytes, added ? 0 : PART_LAUNCH_NS);
    };
    const auto key_parts = [&](bool added) { return worth((k_len + key_block - 1) / key_block * units, query_steps, 21, 2 * keys * row_bytes, added); };
    // Without dropout, whose random numbers neighbouring queries share, the queries of a group's heads are
    // packed where at least two heads' fit a block: 64 x 8 groups of 4 heads of one query over 4096 keys of
    // 128 195 us, each head on its own 415; of 33 queries (8 x 8 groups) 55 and 70.
    p.packed = !drop && group > 1 && 2 * q_len <= ATTENTION_QUERIES;
    const uint64_t forward_blocks = p.packed ? (group * q_len + ATTENTION_QUERIES - 1) / ATTENTION_QUERIES * units : query_blocks;
    p.fine = rows <= FINE_PAIRS / (k_len ? k_len : 1);
    p.forward_parts = worth(forward_blocks, key_steps, 12, rows * (row_bytes + 8), false);
    p.key_parts = key_parts(false);
    p.query_parts = worth(query_blocks, key_steps, 17, rows * row_bytes, p.key_parts > 1);
    if (p.query_parts > 1) p.key_parts = key_parts(true);
    p.forward_groups = forward_blocks * p.forward_parts;
    p.query_groups = query_blocks * p.query_parts;
    p.key_groups = (k_len + key_block - 1) / key_block * units * p.key_parts;
    const auto round = [](uint64_t n) { return (size_t)((n + 255) & ~255ull); };
    p.forward_bytes = p.forward_parts > 1 ? round(p.forward_parts * rows * (p.dim + 2) * sizeof(float)) : 0;
    p.rows_at = 0;
    p.dq_at = round(rows * 2 * sizeof(float));
    p.dkv_at = p.dq_at + (p.query_parts > 1 ? round(p.query_parts * rows * p.dim * sizeof(float)) : 0);
    p.bytes = p.dkv_at + (p.key_parts > 1 ? round(2 * p.key_parts * keys * p.dim * sizeof(float)) : 0);
    return p;
}

// Strides of a tensor of these sizes; one that is never taken may be anything.  Rows do not overlap: a
// fetch's bounds, in bytes, are what keeps it from rows past the last.  An input may have sequences or heads in
// the same memory, an output may not.
static bool strides(const uint64_t (&s)[3], bool output, uint32_t batch, uint32_t length, uint32_t heads, uint32_t head_dim, Strides& to) {
    to = {batch > 1 ? s[0] : 0, length > 1 ? s[1] : head_dim, heads > 1 ? s[2] : 0};
    for (uint64_t n : {to.batch, to.row, to.head})
        if (n % 8 || n > (1ull << 40)) return false;
    if (output && ((batch > 1 && to.batch < head_dim) || (heads > 1 && to.head < head_dim))) return false;
    return to.row >= head_dim && to.row <= (1u << 24);        // a tile's offsets fit 32 bits
}

bool attention_args(const okt_attention* op, bool backward, AttentionArgs& a) {
    if (!op || (op->dtype != OKT_BF16 && op->dtype != OKT_F16)) return false;
    if (op->kv_heads == 0 || op->heads == 0 || op->heads % op->kv_heads) return false;
    if ((uint64_t)op->batch * op->heads > (1u << 20) || op->q_len > (1u << 24) || op->k_len > (1u << 24)) return false;
    if (op->head_dim == 0 || op->head_dim > 128 || op->head_dim % 8) return false;
    if (!(op->scale > 0.0f) || op->scale > 3.0e38f) return false;
    if (!dropout_rule(op->dropout_p, a.drop)) return false;
    if (a.drop.bar != 65536u && (!op->d_seed || !aligned(op->d_seed, 8))) return false;
    if (!aligned(op->d_q_lens, 4) || !aligned(op->d_k_lens, 4)) return false;
    const auto take = [&](const uint64_t (&from)[3], bool keys, Strides& to, bool output = false) {
        return strides(from, output, op->batch, keys ? op->k_len : op->q_len, keys ? op->kv_heads : op->heads, op->head_dim, to);
    };
    if (!take(op->q_stride, false, a.q) || !take(op->k_stride, true, a.k) || !take(op->v_stride, true, a.v) ||
        !take(op->o_stride, false, a.o, !backward)) return false;
    if (backward && (!take(op->do_stride, false, a.d_o) || !take(op->dq_stride, false, a.dq, true) ||
                     !take(op->dk_stride, true, a.dk, true) || !take(op->dv_stride, true, a.dv, true))) return false;
    a.batch = op->batch;
    a.heads = op->heads;
    a.kv_heads = op->kv_heads;
    a.group = op->heads / op->kv_heads;
    a.by_kv = divider(op->kv_heads);
    a.q_len = op->q_len;
    a.k_len = op->k_len;
    a.head_dim = op->head_dim;
    a.site = op->site;
    a.causal = op->causal != 0;
    a.scale = op->scale;
    a.scale_log2 = (float)((double)op->scale * 1.4426950408889634);
    a.seed = op->d_seed;
    a.q_lens = op->d_q_lens;
    a.k_lens = op->d_k_lens;
    return true;
}

}  // namespace okt

extern "C" {

size_t okt_attention_workspace_bytes(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t q_len, uint32_t k_len,
                                     uint32_t head_dim) {
    size_t need = 256;
    for (bool drop : {false, true}) {
        const okt::AttentionPlan plan = okt::attention_plan(batch, heads, kv_heads, q_len, k_len, head_dim, drop);
        for (size_t n : {plan.forward_bytes, plan.bytes}) need = n > need ? n : need;
    }
    return need;
}

int okt_attention_forward(const okt_attention* op, const void* d_q, const void* d_k, const void* d_v, void* d_o_out,
                          float* d_lse_out, void* d_ws, size_t ws_bytes, void* stream) {
    using namespace okt;
    AttentionArgs a;
    if (!attention_args(op, false, a)) return OKT_ERR_INVALID_ARG;
    if (a.batch == 0 || a.q_len == 0) return OKT_OK;
    if (!d_q || !d_o_out || (a.k_len && (!d_k || !d_v))) return OKT_ERR_INVALID_ARG;
    if (!aligned(d_q, 16) || !aligned(d_k, 16) || !aligned(d_v, 16) || !aligned(d_o_out, 16) || !aligned(d_lse_out, 4)) return OKT_ERR_INVALID_ARG;
    const AttentionPlan plan = attention_plan(a.batch, a.heads, a.kv_heads, a.q_len, a.k_len, a.head_dim, a.drop.bar != 65536u);
    if (plan.forward_groups > LAUNCH_GROUPS) return OKT_ERR_INVALID_ARG;
    if (plan.forward_bytes && (!d_ws || !aligned(d_ws, 256) || ws_bytes < plan.forward_bytes)) return OKT_ERR_WORKSPACE;
    for (const void* in : {d_q, a.k_len ? d_k : nullptr, a.k_len ? d_v : nullptr})
        if (same_place(d_o_out, in, a.head_dim)) return OKT_ERR_INVALID_ARG;
    const hipStream_t s = (hipStream_t)stream;
    return op->dtype == OKT_BF16 ? launch_forward_shape<__bf16>(a, plan, d_q, d_k, d_v, d_o_out, d_lse_out, d_ws, s)
                                 : launch_forward_shape<_Float16>(a, plan, d_q, d_k, d_v, d_o_out, d_lse_out, d_ws, s);
}

}  // extern "C"
