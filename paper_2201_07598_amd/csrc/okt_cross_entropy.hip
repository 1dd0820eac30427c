// okt_cross_entropy_forward / _backward: softmax cross entropy of s = h W' + b over a vocabulary, and its gradient, without the logits.
//
//   loss_n = lse_n - s_ny,  lse_n = log sum_v exp s_nv,    d_nv = g_n (exp(s_nv - lse_n) - [v = y_n])
//   dh = d W,  dW = d' h,  db_v = sum_n d_nv
//
// Rows without a label take no part: the others' numbers are listed first, their h copied side by side (and padded to whole tiles
// with zeros), and every later kernel works on the list, whose length it reads from device memory.  With 15 % of the rows labelled
// that is 15 % of the work.
//
// Forward, a tile of logits is a matrix product whose epilogue leaves the largest and the sum of exponentials of its part of a row; a
// second kernel joins a row's parts.  Backward the logits are made again, a piece of the vocabulary at a time, and leave the
// epilogue as d, rounded to the tensors' type, in the workspace; two more products take it from there.  dW of a piece is final; dh
// is summed over the pieces in fp32.  Both passes together make four products where a kept matrix of logits would need three.
//
// d is taken times a factor that makes the largest |g| a power of two, and the sums times its reciprocal: the gradient of a mean is one
// number for all rows, and its rounding, the same in every entry, would be an error of the whole result (the largest entry of a row is
// the label's, g (p - 1), and p - 1 itself loses nothing where p is small).  In fp16 that power is 2^15: g is one
// over the number of rows and p one over the vocabulary's size, and fp16 ends at 2^-24.
//
// The matrix units bound the large sizes, at the clock that their power leaves: 8192 rows x 4096 x 128000 bf16 take 6.4 ms forward
// (1.34 PFLOP/s) and 20.0 backward (three products, 1.29: logits 1.31, dh 1.37, dW, of whose operands both have to be turned, 1.24).  15 % of
// 16384 rows x 1024 x 30522 with a bias: 149 to 165 us forward, of which the launches before and behind the product are 15 to 20, and 470 to 488
// backward, 511 with dW in fp32.  One row to a few hundred: W's way from memory, and two launches (125 x 776 x 10007 fp16 15 us).
#include <algorithm>
#include <math.h>

#include "okt_product.h"

namespace okt {

constexpr uint32_t CE_PAD = 256;                                     // rows, and columns of a piece, are padded to the largest tile
constexpr uint64_t CE_PIECE_BYTES = 1ull << 30;                    // of d in the workspace
constexpr uint32_t CE_SPLIT_TILES = 256;                             // of a gradient, with the parts that its sum is dealt to where tiles are fewer
constexpr uint32_t CE_SPLIT_PIECES = 8;                              // pieces of k that a part has at least: fewer are not worth their sums' way
constexpr uint32_t CE_FINE_ROWS = 256;                               // up to so many, d goes into the second products in two parts (256 x 4096 x 128000 1776 us, 300 rows, in one, 1515)
constexpr uint32_t CE_MAX = 1u << 22;                                // rows, vocabulary
constexpr uint32_t CE_MAX_WIDTH = 1u << 15;
constexpr int CE_THREADS = 256;
constexpr float LOG2E = 1.44269504088896340736f;

typedef ProductShape<4, 2, 2, 4, 2> Large;                           // 256 x 256, one workgroup of eight waves a CU
typedef ProductShape<2, 2, 2, 2, 2> Narrow;                          // 128 x 128, two workgroups a CU: many tiles of a short sum
typedef ProductShape<2, 2, 2, 2, 3> Small;                           // 128 x 128, four waves and two pieces on their way
// The same by eight waves, for logits: two a SIMD wait for LDS in turn (125 x 776 x 10007: 17.0 -> 16.2 us).  The second products, whose
// sums over k are dealt to more workgroups, gain little by it and lose where LDS bounds them (78 x 136 x 143, gradient: 20.9 -> 20.5;
// 700 x 1024 x 3000 46.0 -> 48.5).
typedef ProductShape<2, 1, 2, 4, 3> Spread;
typedef ProductShape<1, 1, 2, 4, 3> Thin;                            // 64 x 128

struct CeHeader { uint32_t count; float raise, lower; uint32_t pad; };

struct CeArgs {
    uint32_t rows, width, vocab, rows_pad, width_pad;
    uint64_t h_stride, weight_stride, dh_stride, dweight_stride;
    uint32_t dloss_step;
    const float* bias;
    const int64_t* labels;
    // workspace
    CeHeader* header;
    float2* counts;                                                  // of every block: labelled rows (as bits), largest finite |g|
    uint32_t* list;                                                  // numbers of the labelled rows
    int32_t* label_of;                                               // of listed row n
    void* h;                                                         // [rows_pad][width_pad]
    float* stats;                                                    // forward: [parts][rows_pad][2], see ce_stats_columns
    float* said;                                                     // forward: s_ny
    float *lse_of, *g_of;                                            // backward, of listed row n
    void* d;                                                         // [rows_pad][piece]
    void* d_rest;                                                    // [CE_FINE_ROWS][piece]: what d's rounding left off
    float* dw_sums;                                                  // [parts][columns of whole tiles][width_pad]
    float* dh_sums;                                                  // [parts][rows of whole tiles][width_pad]
    float* dbias_sums;                                               // [parts][vocab_pad], see ce_dbias_rows
    uint32_t piece, vocab_pad;
    uint32_t logit_tile_n, logit_parts_n;                            // rows of a tile of logits, and parts they leave of the bias's gradient
    __device__ __forceinline__ uint32_t dbias_parts(uint32_t count) const { return (count + logit_tile_n - 1) / logit_tile_n * logit_parts_n; }
};

// ------------------------------------------------------------------ the list of labelled rows

constexpr uint32_t CE_BLOCK = 256;                                   // rows that a thread each counts
constexpr uint32_t CE_GATHERED = 8;                                  // rows that a workgroup gathers
constexpr uint32_t CE_DIRECT = 2048;                                 // up to so many rows, every workgroup counts all of them by itself

__device__ __forceinline__ bool labelled(int64_t y, uint32_t vocab) { return y >= 0 && y < (int64_t)vocab; }

struct CeCount { uint32_t before, all; float top; };                 // labelled rows, and the largest finite |g| of those

__device__ __forceinline__ CeCount count_together(CeCount c, CeCount (&waves)[CE_THREADS / WAVE]) {
#pragma unroll
    for (int m = 1; m < WAVE; m <<= 1) {
        c.before += __shfl_xor(c.before, m, WAVE);
        c.all += __shfl_xor(c.all, m, WAVE);
        c.top = fmaxf(c.top, __shfl_xor(c.top, m, WAVE));
    }
    if (threadIdx.x % WAVE == 0) waves[threadIdx.x / WAVE] = c;
    __syncthreads();
    c = waves[0];
#pragma unroll
    for (int w = 1; w < CE_THREADS / WAVE; ++w) {
        c.before += waves[w].before;
        c.all += waves[w].all;
        c.top = fmaxf(c.top, waves[w].top);
    }
    return c;
}

__device__ __forceinline__ CeCount count_row(const CeArgs& a, const float* dloss, uint64_t row, uint64_t first) {
    if (row >= a.rows || !labelled(a.labels[row], a.vocab)) return {0, 0, 0.0f};
    const float g = dloss ? fabsf(dloss[row * a.dloss_step]) : 0.0f;
    return {row < first ? 1u : 0u, 1u, g < __builtin_inff() ? g : 0.0f};      // what is not finite is its own row's alone
}

__device__ __forceinline__ void add_to(CeCount& c, const CeCount& more) {
    c.before += more.before;
    c.all += more.all;
    c.top = fmaxf(c.top, more.top);
}

// Labelled rows of every block.
__global__ __launch_bounds__(CE_THREADS) void cross_entropy_count_kernel(CeArgs a, const float* dloss) {
    __shared__ CeCount waves[CE_THREADS / WAVE];
    const CeCount c = count_together(count_row(a, dloss, (uint64_t)blockIdx.x * CE_BLOCK + threadIdx.x, 0), waves);
    if (threadIdx.x == 0) a.counts[blockIdx.x] = make_float2(__uint_as_float(c.all), c.top);
}

// Eight rows a workgroup: those with a label go side by side into the workspace, behind all labelled ones before them; the others
// get their zeros.  Zeros fill the last tile, too.
template <typename T>
__global__ __launch_bounds__(CE_THREADS) void cross_entropy_gather_kernel(CeArgs a, const T* h, float* loss, const float* lse_in, float* lse_out,
                                                                              const float* dloss, T* dh) {
    typedef typename Eight<T>::vec vec;
    __shared__ CeCount waves[CE_THREADS / WAVE];
    const uint64_t first = (uint64_t)blockIdx.x * CE_GATHERED;
    const uint32_t lane = threadIdx.x % WAVE, wave = uniform(threadIdx.x / WAVE);
    CeCount c = {0, 0, 0.0f};
    if (a.rows <= CE_DIRECT) {
        for (uint32_t r = threadIdx.x; r < a.rows; r += CE_THREADS) add_to(c, count_row(a, dloss, r, first));
    } else {
        const uint64_t block = first / CE_BLOCK;
        for (uint64_t b = threadIdx.x; b * CE_BLOCK < a.rows; b += CE_THREADS) {
            const float2 v = a.counts[b];
            const uint32_t n = __float_as_uint(v.x);
            add_to(c, {b < block ? n : 0u, n, v.y});
        }
        c.before += count_row(a, nullptr, block * CE_BLOCK + threadIdx.x, first).before;
    }
    c = count_together(c, waves);
    if (blockIdx.x == 0 && threadIdx.x == 0) {
        int e = 0;                                                   // top = half 2^(e - 1), half in [1, 2)
        const bool use = c.top > 0.0f;
        const float half = use ? 2.0f * frexpf(c.top, &e) : 1.0f;
        const int by = use && __is_same(T, _Float16) ? min(16 - e, 120) : 0;
        *a.header = {c.all, ldexpf(1.0f / half, by), ldexpf(half, -by), 0};
    }
    // the labels at once; a wave takes two rows, whose vectors are on their way together
    const bool inside = lane < CE_GATHERED && first + lane < a.rows;
    const int64_t y = inside ? a.labels[first + lane] : -1;
    const uint64_t listed = __ballot(labelled(y, a.vocab));
    constexpr int EACH = CE_GATHERED / (CE_THREADS / WAVE);
    const T* from[EACH];
    T* to[EACH];
#pragma unroll
    for (int q = 0; q < EACH; ++q) {
        const uint32_t i = wave * EACH + q;
        const uint64_t row = first + i;
        const uint32_t n = c.before + __popcll(listed & ((1ull << i) - 1));
        from[q] = listed >> i & 1 ? h + row * a.h_stride : nullptr;
        to[q] = from[q] ? (T*)a.h + (uint64_t)n * a.width_pad : row < a.rows && dh ? dh + row * a.dh_stride : nullptr;
        if (row >= a.rows || lane != i) continue;
        if (from[q]) {
            a.list[n] = (uint32_t)row;
            a.label_of[n] = (int32_t)y;
            if (dloss) {
                a.lse_of[n] = lse_in[row];
                a.g_of[n] = dloss[row * a.dloss_step];
            }
        } else if (loss) {
            loss[row] = 0.0f;
            if (lse_out) lse_out[row] = 0.0f;
        }
    }
#pragma unroll 2
    for (uint32_t x = lane * 8; x < a.width_pad; x += WAVE * 8) {
        vec v[EACH];
#pragma unroll
        for (int q = 0; q < EACH; ++q) {
            v[q] = vec{};
            if (from[q] && x < a.width) v[q] = *reinterpret_cast<const vec*>(from[q] + x);
        }
#pragma unroll
        for (int q = 0; q < EACH; ++q)
            if (to[q] && (from[q] || x < a.width)) *reinterpret_cast<vec*>(to[q] + x) = v[q];
    }
    const uint32_t end = (c.all + CE_PAD - 1) / CE_PAD * CE_PAD;
    for (uint32_t z = c.all + blockIdx.x * (CE_THREADS / WAVE) + wave; z < end; z += gridDim.x * (CE_THREADS / WAVE)) {
        for (uint32_t x = lane * 8; x < a.width_pad; x += WAVE * 8) *reinterpret_cast<vec*>((T*)a.h + (uint64_t)z * a.width_pad + x) = vec{};
        if (lane == 0) {
            a.label_of[z] = -1;
            if (dloss) a.lse_of[z] = a.g_of[z] = 0.0f;
        }
    }
}

// ------------------------------------------------------------------ logits

// What is added to a tile's logits, in LDS: the bias, -infinity past the vocabulary.
template <class S>
__device__ __forceinline__ void load_bias(float* tile, const CeArgs& a, uint32_t v) {
    for (uint32_t i = threadIdx.x; i < S::TILE_M; i += S::THREADS) tile[i] = v + i >= a.vocab ? -__builtin_inff() : a.bias ? a.bias[v + i] : 0.0f;
}

// Logits of a lane's row of column n of the wave's squares; `part`: the wave's part of that tile.
template <class S>
__device__ __forceinline__ void logits_of_row(float (&s)[S::MT * 16], const f32x16 (&c)[S::MT][S::NT], int n, const float* part, bool biased) {
#pragma unroll
    for (int m = 0; m < S::MT; ++m)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[m * 16 + r] = c[m][n][r];
    if (!biased) return;
#pragma unroll
    for (int m = 0; m < S::MT; ++m)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const float4 b = *reinterpret_cast<const float4*>(part + m * 32 + threadIdx.x % WAVE / 32 * 16 + q * 4);
            s[m * 16 + 4 * q] += b.x;
            s[m * 16 + 4 * q + 1] += b.y;
            s[m * 16 + 4 * q + 2] += b.z;
            s[m * 16 + 4 * q + 3] += b.w;
        }
}

template <typename T, class S> using LogitProduct = Product<T, S, KMajor<T, S::TILE_M, S::WAVES, true>, KMajor<T, S::TILE_N, S::WAVES, false>>;

// Of the tile that begins at vocabulary v and listed row n.
template <typename T, class S>
__device__ __forceinline__ LogitProduct<T, S> logits_at(const CeArgs& a, const T* weight, uint32_t v, uint32_t n, const char* lds) {
    const T* h = (const T*)a.h;
    return LogitProduct<T, S>(
        {weight + v * a.weight_stride, weight + (a.vocab - 1) * a.weight_stride + a.width, (uint32_t)(a.weight_stride * 2)},
        {h + (uint64_t)n * a.width_pad, h + (uint64_t)a.rows_pad * a.width_pad, a.width_pad * 2}, a.width, lds);
}

// What a lane has to know of its rows; fetched before the next tile's operands are, behind which it would arrive.
template <class S>
struct RowFacts {
    uint32_t label[S::NT];
    float g[S::NT], lse[S::NT];
    __device__ __forceinline__ explicit RowFacts(const uint32_t* labels) {
#pragma unroll
        for (int n = 0; n < S::NT; ++n) label[n] = labels[n * 32];
    }
    __device__ __forceinline__ RowFacts(const CeArgs& a, uint32_t row, bool backward) {
#pragma unroll
        for (int n = 0; n < S::NT; ++n) {
            label[n] = (uint32_t)a.label_of[row + n * 32];
            if (backward) {
                g[n] = a.g_of[row + n * 32];
                lse[n] = a.lse_of[row + n * 32];
            }
        }
    }
};

// Where a workgroup has a CU for itself it stays, and the next tile's first operands are on their way while this one's logits are
// worked on (2458 rows x 1024 x 30522: 164 -> 157 us; small tiles, of which there are few, gain nothing and lose 1.4 us).
template <class S> constexpr bool STAYS = S::TILE_M == 256;

// Tiles of logits; `finish` is called with a tile's sums, its place, its bias and its rows' facts.
template <typename T, class S, bool BACKWARD, class F>
__device__ __forceinline__ void logit_tiles(const CeArgs& a, const T* weight, uint32_t from, uint32_t columns, const F& finish) {
    __shared__ __attribute__((aligned(1024))) char lds[S::BYTES];
    __shared__ float bias[2][S::TILE_M];
    const uint32_t count = uniform(a.header->count), tiles_m = (columns + S::TILE_M - 1) / S::TILE_M, tiles_n = (count + S::TILE_N - 1) / S::TILE_N;
    uint32_t group = blockIdx.x;
    TilePlace tile = tile_place(group, tiles_m, tiles_n);
    if (!tile.there) return;
    LogitProduct<T, S> p = logits_at<T, S>(a, weight, from + tile.m * S::TILE_M, tile.n * S::TILE_N, lds);
    p.begin();
    load_bias<S>(bias[0], a, from + tile.m * S::TILE_M);
    for (uint32_t turn = 0; ; ++turn) {
        f32x16 c[S::MT][S::NT];
        clear<S>(c);
        p.run(c, lds);
        const uint32_t at = tile.m * S::TILE_M + S::wave_m() * (S::MT * 32), part_n = tile.n * S::WN + S::wave_n();
        const RowFacts<S> facts(a, part_n * (S::NT * 32) + threadIdx.x % 32, BACKWARD);
        __builtin_amdgcn_sched_barrier(0);
        group += gridDim.x;
        const TilePlace next = STAYS<S> ? tile_place(group, tiles_m, tiles_n) : TilePlace{0, 0, false};
        if (next.there) {
            p = logits_at<T, S>(a, weight, from + next.m * S::TILE_M, next.n * S::TILE_N, lds);
            p.begin();
            load_bias<S>(bias[(turn + 1) % 2], a, from + next.m * S::TILE_M);
        }
        __builtin_amdgcn_sched_barrier(0);
        finish(c, at, part_n, bias[turn % 2] + S::wave_m() * (S::MT * 32), facts, count);
        if (!next.there) return;
        tile = next;
    }
}

// What a tile of logits leaves: the largest and the sum of exponentials of its part of a row, and the label's logit.
template <class S>
__device__ __forceinline__ void part_of_rows(const CeArgs& a, const f32x16 (&c)[S::MT][S::NT], uint32_t v0, uint32_t part_n, const float* bias,
                                             const RowFacts<S>& facts, uint32_t count) {
    const uint32_t lane = threadIdx.x % WAVE, part = v0 / (S::MT * 32);
    const bool biased = a.bias || v0 + S::MT * 32 > a.vocab;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        const uint32_t row = part_n * (S::NT * 32) + n * 32 + lane % 32;
        float s[S::MT * 16];
        logits_of_row<S>(s, c, n, bias, biased);
        float top = -__builtin_inff();
#pragma unroll
        for (int i = 0; i < S::MT * 16; ++i) top = fmaxf(top, s[i]);
        top = max_halves(top);
        // the largest is taken off first: off a rounded product with log2 e, its own exponential would not be 1 and a sure row's loss not 0
        const float base = top == -__builtin_inff() ? 0.0f : top;
        float sum = 0.0f;
#pragma unroll
        for (int i = 0; i < S::MT * 16; ++i) sum += __builtin_amdgcn_exp2f((s[i] - base) * LOG2E);
        sum = sum_halves(sum);
        if (lane < 32 && row < count)
            *reinterpret_cast<float2*>(a.stats + ((uint64_t)part * a.rows_pad + row) * 2) = make_float2(top, sum);
        const uint32_t mine = facts.label[n] - v0 - lane / 32 * 16;      // far above a wave's part where it is none of its
        if (__ballot(mine < S::MT * 32u)) {
#pragma unroll
            for (int m = 0; m < S::MT; ++m)
#pragma unroll
                for (int r = 0; r < 16; ++r)
                    if (mine == m * 32u + r) a.said[row] = s[m * 16 + r];
        }
    }
}

template <typename T, class S>
__global__ __launch_bounds__(S::THREADS) void cross_entropy_forward_kernel(CeArgs a, const T* weight) {
    logit_tiles<T, S, false>(a, weight, 0, a.vocab, [&](const f32x16 (&c)[S::MT][S::NT], uint32_t v0, uint32_t part_n, const float* bias,
                                                        const RowFacts<S>& facts, uint32_t count) {
        part_of_rows<S>(a, c, v0, part_n, bias, facts, count);
    });
}

// Few rows, of few tiles, are taken as they lie: every workgroup lists the labelled ones by itself and fetches its tile's by their numbers, so nothing
// is laid side by side first (125 x 776 x 10007: 20.4 -> 17.0 us, 481 x 80 x 2048 14.1 -> 11.1).  The first one writes the list and the other rows' zeros.
template <typename T, class S>
__global__ __launch_bounds__(S::THREADS) void cross_entropy_direct_kernel(CeArgs a, const T* h, const T* weight, float* loss, float* lse) {
    typedef Product<T, S, KMajor<T, S::TILE_M, S::WAVES, true>, ListedRows<T, S::TILE_N, S::WAVES>> Logits;
    constexpr uint32_t CHUNKS = CE_DIRECT / S::THREADS;
    static_assert(CHUNKS * S::THREADS == CE_DIRECT && CHUNKS * S::WAVES <= WAVE && S::THREADS >= S::TILE_N, "");
    __shared__ __attribute__((aligned(1024))) char lds[S::BYTES];
    __shared__ float bias[S::TILE_M];
    __shared__ uint32_t counts[WAVE], row_of[S::TILE_N], label_of[S::TILE_N];
    const uint32_t lane = threadIdx.x % WAVE, wave = uniform(threadIdx.x / WAVE);
    int64_t y[CHUNKS];
#pragma unroll
    for (uint32_t k = 0; k < CHUNKS; ++k) {
        const uint32_t row = k * S::THREADS + threadIdx.x;
        y[k] = row < a.rows ? a.labels[row] : -1;
    }
    if (threadIdx.x < WAVE) counts[threadIdx.x] = 0;
    if (threadIdx.x < S::TILE_N) row_of[threadIdx.x] = label_of[threadIdx.x] = NO_ROW;
    __syncthreads();
    uint64_t listed[CHUNKS];                                         // lanes whose row has a label
#pragma unroll
    for (uint32_t k = 0; k < CHUNKS; ++k) {
        listed[k] = __ballot(labelled(y[k], a.vocab));
        if (lane == 0) counts[k * S::WAVES + wave] = __popcll(listed[k]);
    }
    __syncthreads();
    const uint32_t up_to = wave_inclusive_scan_u32(counts[lane]), count = uniform(__shfl(up_to, WAVE - 1, WAVE));
    const TilePlace tile = tile_place(blockIdx.x, (a.vocab + S::TILE_M - 1) / S::TILE_M, (count + S::TILE_N - 1) / S::TILE_N);
    const bool writes = blockIdx.x == 0;
    if (!tile.there && !writes) return;
#pragma unroll
    for (uint32_t k = 0; k < CHUNKS; ++k) {
        const uint32_t row = k * S::THREADS + threadIdx.x, group = k * S::WAVES + wave;
        const uint32_t before = group ? __shfl(up_to, group - 1, WAVE) : 0;
        const uint32_t n = before + __popcll(listed[k] & ((1ull << lane) - 1));
        if (listed[k] >> lane & 1) {
            if (tile.there && n / S::TILE_N == tile.n) {
                row_of[n % S::TILE_N] = row;
                label_of[n % S::TILE_N] = (uint32_t)y[k];
            }
            if (writes) a.list[n] = row;
        } else if (writes && row < a.rows) {
            loss[row] = 0.0f;
            if (lse) lse[row] = 0.0f;
        }
    }
    if (writes && threadIdx.x == 0) *a.header = {count, 1.0f, 1.0f, 0};
    if (!tile.there) return;
    const uint32_t v = tile.m * S::TILE_M;
    load_bias<S>(bias, a, v);
    __syncthreads();
    Logits p({weight + v * a.weight_stride, weight + (a.vocab - 1) * a.weight_stride + a.width, (uint32_t)(a.weight_stride * 2)},
             {h, h + (a.rows - 1) * a.h_stride + a.width, (uint32_t)(a.h_stride * 2), row_of}, a.width, lds);
    f32x16 c[S::MT][S::NT];
    clear<S>(c);
    p.begin();
    p.run(c, lds);
    const uint32_t in_tile = S::wave_n() * (S::NT * 32);
    part_of_rows<S>(a, c, v + S::wave_m() * (S::MT * 32), tile.n * S::WN + S::wave_n(), bias + S::wave_m() * (S::MT * 32),
                    RowFacts<S>(label_of + in_tile + lane % 32), count);
}

// Sixteen rows a workgroup, and 64 threads a row, each every 64th part.
constexpr int CE_JOIN_THREADS = 1024;
struct RowSum { float top, sum; };
__device__ __forceinline__ RowSum together(RowSum x, RowSum y) {
    const float top = fmaxf(x.top, y.top);
    if (top == -__builtin_inff()) return {top, x.sum + y.sum};      // 0, or NaN
    return {top, x.sum * __builtin_amdgcn_exp2f((x.top - top) * LOG2E) + y.sum * __builtin_amdgcn_exp2f((y.top - top) * LOG2E)};
}

__global__ __launch_bounds__(CE_JOIN_THREADS) void cross_entropy_join_kernel(CeArgs a, uint32_t parts, float* loss, float* lse) {
    __shared__ RowSum waves[CE_JOIN_THREADS / WAVE][16];
    const uint32_t count = uniform(a.header->count), r = threadIdx.x % 16, share = threadIdx.x / 16, row = blockIdx.x * 16 + r;
    if (blockIdx.x * 16 >= count) return;
    RowSum v = {-__builtin_inff(), 0.0f};
    const bool last = threadIdx.x < 16 && row < count;               // has the row's sum in the end
    const uint32_t to = last ? a.list[row] : 0;
    const float said = last ? a.said[row] : 0.0f;
    if (row < count)
#pragma unroll 4
        for (uint32_t p = share; p < parts; p += CE_JOIN_THREADS / 16) {
            const float2 t = *reinterpret_cast<const float2*>(a.stats + ((uint64_t)p * a.rows_pad + row) * 2);
            v = together(v, {t.x, t.y});
        }
    const auto lanes = [&](RowSum x) {                               // the four shares of a wave
#pragma unroll
        for (int m = 16; m < WAVE; m <<= 1) x = together(x, {__shfl_xor(x.top, m, WAVE), __shfl_xor(x.sum, m, WAVE)});
        return x;
    };
    v = lanes(v);
    if (threadIdx.x % WAVE < 16) waves[threadIdx.x / WAVE][r] = v;
    __syncthreads();
    if (threadIdx.x >= WAVE) return;
    v = waves[share][r];
#pragma unroll
    for (int k = 4; k < CE_JOIN_THREADS / WAVE; k += 4) v = together(v, waves[k + share][r]);
    v = lanes(v);
    if (!last) return;
    const float all = v.top == -__builtin_inff() && v.sum == 0.0f ? v.top : v.top + logf(v.sum);
    loss[to] = all - said;
    if (lse) lse[to] = all;
}

// ------------------------------------------------------------------ the gradient of the logits

// Sums over the 32 lanes of a half of N values each; lane l % 32 gets those of values N (l % 32) / 32 on (of 16 values two lanes the same).  Every step hands over the half of the
// values that the other lane goes on with, so all steps together cost two exchanges a value and not five.
template <int N>
__device__ __forceinline__ void sums_over_lanes(float (&v)[N]) {
    static_assert(N == 64 || N == 32 || N == 16, "");
#pragma unroll
    for (int i = 0; i < N / 2; ++i) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[i]), __float_as_uint(v[i + N / 2]), false, false);
        v[i] = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
#define OKT_HALVE(KEEP, BIT, CTRL)                                                                                         \
    _Pragma("unroll") for (int i = 0; i < (KEEP); ++i) {                                                                  \
        const bool upper = threadIdx.x & (BIT);                                                                             \
        const float mine = upper ? v[i + (KEEP)] : v[i], theirs = upper ? v[i] : v[i + (KEEP)];                            \
        v[i] = mine + __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(theirs), CTRL, 0xf, 0xf, true));             \
    }
    OKT_HALVE(N / 4, 8, 0x140)        // row_mirror
    OKT_HALVE(N / 8, 4, 0x141)        // row_half_mirror
    OKT_HALVE(N / 16, 2, 0x4E)        // quad_perm [2, 3, 0, 1]
    if constexpr (N >= 32) {
        OKT_HALVE(N / 32, 1, 0xB1)    // quad_perm [1, 0, 3, 2]
    } else {
        v[0] += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v[0]), 0xB1, 0xf, 0xf, true));
    }
#undef OKT_HALVE
}

// d of a piece of the vocabulary that begins at `from`.
template <typename T, class S>
__global__ __launch_bounds__(S::THREADS) void cross_entropy_gradient_kernel(CeArgs a, const T* weight, uint32_t from, uint32_t columns) {
    const float raise = a.header->raise;
    logit_tiles<T, S, true>(a, weight, from, columns, [&](const f32x16 (&c)[S::MT][S::NT], uint32_t at, uint32_t part_n, const float* bias,
                                                          const RowFacts<S>& facts, uint32_t count) {
        const bool fine = count <= CE_FINE_ROWS;
        const uint32_t lane = threadIdx.x % WAVE, v0 = from + at;
        const bool biased = a.bias || v0 + S::MT * 32 > a.vocab;
        float sums[S::MT * 16];
#pragma unroll
        for (int i = 0; i < S::MT * 16; ++i) sums[i] = 0.0f;
#pragma unroll
        for (int n = 0; n < S::NT; ++n) {
            const uint32_t row = part_n * (S::NT * 32) + n * 32 + lane % 32;
            const bool there = row < count;
            const float g = facts.g[n] * raise;
            const uint32_t mine = facts.label[n] - v0 - lane / 32 * 16;
            float s[S::MT * 16];
            logits_of_row<S>(s, c, n, bias, biased);
#pragma unroll
            for (int i = 0; i < S::MT * 16; ++i) s[i] = __builtin_amdgcn_exp2f((s[i] - facts.lse[n]) * LOG2E);
            if (__ballot(mine < S::MT * 32u)) {
#pragma unroll
                for (int m = 0; m < S::MT; ++m)
#pragma unroll
                    for (int r = 0; r < 16; ++r) s[m * 16 + r] -= mine == m * 32u + r ? 1.0f : 0.0f;
            }
            T* to = (T*)a.d + (uint64_t)row * a.piece + at + lane / 32 * 16;
#pragma unroll
            for (int m = 0; m < S::MT; ++m) {
                f32x8 low, high;
#pragma unroll
                for (int r = 0; r < 16; ++r) {
                    const float d = there ? s[m * 16 + r] * g : 0.0f;        // rows behind the last one: zeros, whatever the bias is
                    sums[m * 16 + r] += d;
                    (r < 8 ? low : high)[r % 8] = d;
                }
                store_eight(to + m * 32, low);
                store_eight(to + m * 32 + 8, high);
                if (fine) {
                    const auto rest = [](f32x8 v) { return v - __builtin_convertvector(__builtin_convertvector(v, frag<T>), f32x8); };
                    T* more = (T*)a.d_rest + (uint64_t)row * a.piece + at + lane / 32 * 16 + m * 32;
                    store_eight(more, rest(low));
                    store_eight(more + 8, rest(high));
                }
            }
        }
        if (!a.dbias_sums) return;
        sums_over_lanes(sums);
        constexpr int EACH = S::MT > 1 ? S::MT / 2 : 1;
        const uint32_t first = lane % 32 * (S::MT * 16) / 32;
        float* to = a.dbias_sums + (uint64_t)part_n * a.vocab_pad + v0 + first / 16 * 32 + lane / 32 * 16 + first % 16;
#pragma unroll
        for (int i = 0; i < EACH; ++i) to[i] = sums[i];
    });
}

// ------------------------------------------------------------------ gradients of h, W and the bias

// How many parts a sum over so many pieces of k is dealt to, so that few tiles fill the chip as well.
__host__ __device__ __forceinline__ uint32_t ce_parts(uint32_t tiles, uint32_t pieces) {
    const uint32_t room = CE_SPLIT_TILES / (tiles ? tiles : 1), worth = pieces / CE_SPLIT_PIECES, parts = room < worth ? room : worth;
    return parts ? parts : 1;
}
struct Split { uint32_t tiles_m, tiles_n, parts; };
template <class S>
__device__ __forceinline__ Split ce_split(uint32_t m, uint32_t n, uint32_t k) {
    const uint32_t tiles_m = (m + S::TILE_M - 1) / S::TILE_M, tiles_n = (n + S::TILE_N - 1) / S::TILE_N;
    return {tiles_m, tiles_n, ce_parts(tiles_m * tiles_n, (k + PRODUCT_K - 1) / PRODUCT_K)};
}
// dh: over the vocabulary of a whole piece; dW: over the listed rows.
template <class S> __device__ __forceinline__ Split dh_split(const CeArgs& a, uint32_t count) {
    Split s = ce_split<S>(a.width_pad, count, a.piece);
    if (count <= CE_FINE_ROWS) s.parts = s.parts > 1 ? s.parts / 2 * 2 : 2;          // every other one of d's rest
    return s;
}
template <class S> __device__ __forceinline__ Split dw_split(const CeArgs& a, uint32_t count, uint32_t columns) {
    return ce_split<S>(a.width_pad, columns, a.dw_sums ? count : 0);
}

// A wave's sums as fp32, row by row of n.
template <class S>
__device__ __forceinline__ void store_sums(float* sums, uint32_t width_pad, const f32x16 (&c)[S::MT][S::NT], uint32_t m0, uint32_t n0, uint32_t rows, bool first) {
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        if (n0 + n * 32 >= rows) continue;
        float* to = sums + (uint64_t)(n0 + n * 32) * width_pad + m0;
#pragma unroll
        for (int m = 0; m < S::MT; ++m) {
            if (m0 + m * 32 >= width_pad) continue;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                float4* at = reinterpret_cast<float4*>(to + m * 32 + q * 4);
                float4 v = make_float4(c[m][n][4 * q], c[m][n][4 * q + 1], c[m][n][4 * q + 2], c[m][n][4 * q + 3]);
                if (!first) {
                    const float4 w = *at;
                    v = make_float4(v.x + w.x, v.y + w.y, v.z + w.z, v.w + w.w);
                }
                *at = v;
            }
        }
    }
}

// dh += d W over a piece.  With few rows one entry of d, the label's, is most of a row's gradient, and its rounding would be the row's
// error (up to 2.5 times that of the output's own); so d's rest goes in as well, as further parts of the sum, beside which W comes by once.
template <typename T, class S>
__device__ __forceinline__ void dh_tile(const CeArgs& a, const T* weight, uint32_t from, uint32_t columns, uint32_t group, uint32_t count, char* lds) {
    if (count == 0) return;
    const Split split = dh_split<S>(a, count);
    const TilePlace tile = tile_place(group, split.tiles_m, split.tiles_n * split.parts);
    if (!tile.there) return;
    const uint32_t part = tile.n / split.tiles_n, n_tile = tile.n % split.tiles_n;
    const bool fine = count <= CE_FINE_ROWS, rest = fine && part % 2;
    const uint32_t pieces = (columns + PRODUCT_K - 1) / PRODUCT_K, shares = fine ? split.parts / 2 : split.parts, share = fine ? part / 2 : part;
    const uint32_t k0 = (uint32_t)((uint64_t)pieces * share / shares) * PRODUCT_K, k1 = (uint32_t)((uint64_t)pieces * (share + 1) / shares) * PRODUCT_K;
    const uint32_t col = tile.m * S::TILE_M, row = n_tile * S::TILE_N;
    typedef Transposed<T, S::TILE_M, S::WAVES, true> A;
    typedef KMajor<T, S::TILE_N, S::WAVES, false> B;
    const T *d = rest ? (const T*)a.d_rest : (const T*)a.d, *end = d + (uint64_t)(rest ? CE_FINE_ROWS : a.rows_pad) * a.piece;
    f32x16 c[S::MT][S::NT];
    clear<S>(c);
    Product<T, S, A, B> p(A(weight + (from + k0) * a.weight_stride + col, weight + (a.vocab - 1) * a.weight_stride + a.width, a.weight_stride * 2,
                            a.width - min(a.width, col)),
                          B(d + (uint64_t)row * a.piece + k0, end, a.piece * 2), k1 - k0, lds);
    p.begin();
    p.run(c, lds);
    const uint32_t lane = threadIdx.x % WAVE, m0 = col + S::wave_m() * (S::MT * 32) + lane / 32 * 16, n0 = row + S::wave_n() * (S::NT * 32) + lane % 32;
    store_sums<S>(a.dh_sums + (uint64_t)part * split.tiles_n * S::TILE_N * a.width_pad, a.width_pad, c, m0, n0, count, from == 0);
}

// Eight columns a lane of the sum of a row's parts.
__device__ __forceinline__ f32x8 parts_of_row(const float* sums, uint64_t part_floats, uint32_t parts, uint64_t at) {
    f32x8 sum = 0.0f;
#pragma unroll 8
    for (uint32_t p = 0; p < parts; ++p) sum += load_eight(sums + p * part_floats + at);
    return sum;
}

// dW = d' h over the listed rows, of the vocabulary's piece; its parts as fp32 where there are several.
template <typename T, typename W, class S>
__device__ __forceinline__ void dweight_tile(const CeArgs& a, W* dweight, uint32_t from, uint32_t columns, uint32_t group, uint32_t count, char* lds) {
    const Split split = dw_split<S>(a, count, columns);
    const TilePlace tile = tile_place(group, split.tiles_m, split.tiles_n * split.parts);
    if (!tile.there) return;
    const uint32_t part = tile.n / split.tiles_n, pieces = (count + PRODUCT_K - 1) / PRODUCT_K;
    const uint32_t k0 = (uint32_t)((uint64_t)pieces * part / split.parts) * PRODUCT_K, k1 = (uint32_t)((uint64_t)pieces * (part + 1) / split.parts) * PRODUCT_K;
    const uint32_t col = tile.m * S::TILE_M, v = tile.n % split.tiles_n * S::TILE_N;
    const T* h = (const T*)a.h;
    typedef Transposed<T, S::TILE_M, S::WAVES, true> A;
    typedef Transposed<T, S::TILE_N, S::WAVES, false> B;
    const A rows_of_h(h + (uint64_t)k0 * a.width_pad + col, h + (uint64_t)a.rows_pad * a.width_pad, a.width_pad * 2, a.width_pad - min(a.width_pad, col));
    const auto d_of = [&](const void* d, uint32_t rows) {
        return B((const T*)d + (uint64_t)k0 * a.piece + v, (const T*)d + (uint64_t)rows * a.piece, (uint64_t)a.piece * 2, a.piece - v);
    };
    f32x16 c[S::MT][S::NT];
    clear<S>(c);
    const bool fine = count <= CE_FINE_ROWS;                         // then d's rest stands behind d, beside the same rows again
    Product<T, S, A, B, true> p(rows_of_h, d_of(a.d, a.rows_pad), (k1 - k0) * (fine ? 2 : 1), lds);
    if (fine) {
        p.again = k1 - k0;
        p.again_a = p.a.from;
        p.again_b = d_of(a.d_rest, CE_FINE_ROWS).from;
    }
    p.begin();
    p.run(c, lds);
    const uint32_t lane = threadIdx.x % WAVE, m0 = col + S::wave_m() * (S::MT * 32) + lane / 32 * 16, n0 = v + S::wave_n() * (S::NT * 32) + lane % 32;
    if (split.parts > 1) {
        store_sums<S>(a.dw_sums + (uint64_t)part * split.tiles_n * S::TILE_N * a.width_pad, a.width_pad, c, m0, n0, columns, true);
        return;
    }
    const float lower = a.header->lower;
#pragma unroll
    for (int n = 0; n < S::NT; ++n) {
        if (n0 + n * 32 >= columns) continue;
        W* to = dweight + (from + n0 + n * 32) * a.dweight_stride + m0;
#pragma unroll
        for (int m = 0; m < S::MT; ++m)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                if (m0 + m * 32 + half * 8 >= a.width) continue;
                f32x8 e;
#pragma unroll
                for (int r = 0; r < 8; ++r) e[r] = c[m][n][half * 8 + r] * lower;
                store_eight(to + m * 32 + half * 8, e);
            }
    }
}

// Both gradients of a piece in one launch, dh's workgroups before dW's: the ones fill the CUs that the others leave.
template <typename T, typename W, class S>
__global__ __launch_bounds__(S::THREADS) void cross_entropy_products_kernel(CeArgs a, const T* weight, W* dweight, uint32_t from, uint32_t columns, uint32_t dh_groups) {
    __shared__ __attribute__((aligned(1024))) char lds[S::BYTES];
    const uint32_t count = uniform(a.header->count);
    if (blockIdx.x < dh_groups) dh_tile<T, S>(a, weight, from, columns, blockIdx.x, count, lds);
    else dweight_tile<T, W, S>(a, dweight, from, columns, blockIdx.x - dh_groups, count, lds);
}

// What is left when the products are done: the parts of dh and dW, a wave 512 columns of a row, and of the bias's
// gradient, a thread a column.  Workgroups in this order.
struct CeFinish { uint32_t dh_groups, dw_groups; };                  // behind them the bias's
template <typename T, typename W, class S>
__global__ __launch_bounds__(CE_THREADS) void cross_entropy_finish_kernel(CeArgs a, T* dh, W* dweight, float* dbias, uint32_t from, uint32_t columns, CeFinish f) {
    const uint32_t count = uniform(a.header->count), across = (a.width + WAVE * 8 - 1) / (WAVE * 8);
    const float lower = a.header->lower;
    uint32_t group = blockIdx.x;
    const bool is_dh = group < f.dh_groups;
    if (is_dh || group < f.dh_groups + f.dw_groups) {
        if (!is_dh) group -= f.dh_groups;
        const Split split = is_dh ? dh_split<S>(a, count) : dw_split<S>(a, count, columns);
        if (!is_dh && split.parts == 1) return;
        const uint32_t rows = is_dh ? count : columns, c = (group % across * WAVE + threadIdx.x % WAVE) * 8;
        const uint32_t step = (is_dh ? f.dh_groups : f.dw_groups) / across;
        if (c >= a.width) return;
        for (uint32_t n = group / across * (CE_THREADS / WAVE) + threadIdx.x / WAVE; n < rows; n += step * (CE_THREADS / WAVE)) {
            const f32x8 sum = lower * parts_of_row(is_dh ? a.dh_sums : a.dw_sums, (uint64_t)split.tiles_n * S::TILE_N * a.width_pad, split.parts,
                                                   (uint64_t)n * a.width_pad + c);
            if (is_dh) store_eight(dh + a.list[n] * a.dh_stride + c, sum);
            else store_eight(dweight + (from + n) * a.dweight_stride + c, sum);
        }
        return;
    }
    const uint32_t v = (group - f.dh_groups - f.dw_groups) * CE_THREADS + threadIdx.x;
    if (v >= a.vocab) return;
    const uint32_t parts = a.dbias_parts(count);
    float sum = 0.0f;
#pragma unroll 8
    for (uint32_t p = 0; p < parts; ++p) sum += a.dbias_sums[(uint64_t)p * a.vocab_pad + v];
    dbias[v] = lower * sum;
}

// ------------------------------------------------------------------ host

struct CePlan {
    uint32_t rows_pad, width_pad, vocab_pad, piece;
    bool small_logits, small_products, narrow_products, split_dweight;
    uint64_t logit_groups, piece_groups, dh_groups, dweight_groups;
    size_t counts_at, list_at, label_at, h_at, lse_at, g_at;         // shared and backward
    size_t stats_at, said_at, forward_bytes;
    size_t d_at, rest_at, dh_at, dw_at, dbias_at, backward_bytes;
};

static uint64_t ce_up(uint64_t n, uint64_t by) { return (n + by - 1) / by * by; }

// Tiles of 256 x 256 where they fill the chip, else of 128 x 128, two workgroups a CU; and those for up to 128 rows, of which the others are half
// zeros (x 4096 x 128000, forward: 128 rows 217 us in small tiles, 270 in large ones; 129 rows 329 and 271, 513 785 and 616; 300 x 1024 x 30522 43.7 and 37.2).
static bool ce_small(uint64_t m, uint64_t n) { return n <= 128 || (m + 255) / 256 * ((n + 255) / 256) < 200; }

// The same where a sum over k can be dealt to several workgroups.
static bool ce_small_split(uint64_t m, uint64_t n, uint64_t k) {
    const uint64_t tiles = (m + 255) / 256 * ((n + 255) / 256), parts = k / (PRODUCT_K * CE_SPLIT_PIECES);
    return n <= 128 || tiles * (parts ? parts : 1) < 200;
}

// Columns and rows of the least part of a tile of logits that leaves its sums by itself: what one of its waves has.  (Which of the small tiles are
// taken is seen at the launch.)
static uint32_t ce_stats_columns(bool small) { return 32 * (small ? std::min(Thin::MT, Spread::MT) : Large::MT); }
static uint32_t ce_dbias_rows(bool small) { return 32 * (small ? std::min(Thin::NT, Spread::NT) : Large::NT); }

static bool ce_plan(uint64_t rows, uint32_t width, uint32_t vocab, CePlan& p) {
    if (rows > CE_MAX || vocab == 0 || vocab > CE_MAX || width < 8 || width > CE_MAX_WIDTH || width % 8 != 0) return false;
    const uint64_t some = rows ? rows : 1;
    p.rows_pad = (uint32_t)ce_up(some, CE_PAD);
    p.width_pad = (uint32_t)ce_up(width, PRODUCT_K);
    p.vocab_pad = (uint32_t)ce_up(vocab, CE_PAD);
    uint64_t most = CE_PIECE_BYTES / (2ull * p.rows_pad) / CE_PAD * CE_PAD;
    if (most < 4096) most = 4096;
    const uint64_t pieces = (p.vocab_pad + most - 1) / most;
    p.piece = (uint32_t)ce_up((p.vocab_pad + pieces - 1) / pieces, CE_PAD);
    const auto tiles = [](uint64_t n, bool small) { return (n + (small ? 127 : 255)) / (small ? 128 : 256); };
    p.small_logits = ce_small(vocab, some);
    p.small_products = ce_small_split(p.width_pad, some, p.piece) && ce_small_split(p.width_pad, p.piece, some);
    p.logit_groups = tile_groups(tiles(vocab, p.small_logits) * tiles(some, p.small_logits));
    p.piece_groups = tile_groups(tiles(p.piece, p.small_logits) * tiles(some, p.small_logits));
    if (p.logit_groups > UINT32_MAX / 2) return false;
    // few rows, for which dW is much to write and little to sum (10 x 256 x 100000: 108 -> 83 to 87 us, 100 x 4096 x 60000 628 -> 552 to 574;
    // 45 x 1632 x 2982, with few tiles, would go from 42 to 50)
    p.narrow_products = some <= CE_FINE_ROWS && tiles(p.width_pad, true) * tiles(p.piece, true) > 1024;
    if (p.narrow_products) p.small_products = true;
    const uint64_t across = tiles(p.width_pad, p.small_products), dh_tiles = across * tiles(some, p.small_products);
    const uint64_t dw_tiles = across * tiles(p.piece, p.small_products);
    const uint64_t fine_tiles = 2 * across * tiles(some < CE_FINE_ROWS ? some : CE_FINE_ROWS, p.small_products);
    p.dh_groups = tile_groups(dh_tiles > CE_SPLIT_TILES ? dh_tiles : CE_SPLIT_TILES);
    if (p.dh_groups < fine_tiles) p.dh_groups = tile_groups(fine_tiles);
    p.dweight_groups = tile_groups(dw_tiles > CE_SPLIT_TILES ? dw_tiles : CE_SPLIT_TILES);
    // the last piece of the vocabulary, with fewer tiles, may be split where the others are not
    const uint64_t least = across * tiles(pieces > 1 ? 1 : vocab, p.small_products);
    p.split_dweight = least <= CE_SPLIT_TILES && ce_parts((uint32_t)least, (uint32_t)((some + PRODUCT_K - 1) / PRODUCT_K)) > 1;
    for (const uint64_t groups : {p.small_logits ? p.logit_groups : 0, p.dh_groups, p.dweight_groups})
        if (groups > LAUNCH_GROUPS / 2) return false;
    size_t at = 256;
    const auto place = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 255) / 256 * 256;
        return here;
    };
    p.counts_at = place(8ull * (p.rows_pad / CE_BLOCK));
    p.list_at = place(4ull * p.rows_pad);
    p.label_at = place(4ull * p.rows_pad);
    p.h_at = place(2ull * p.rows_pad * p.width_pad);
    const size_t shared = at;
    p.stats_at = place(8ull * p.rows_pad * (p.vocab_pad / ce_stats_columns(p.small_logits)));
    p.said_at = place(4ull * p.rows_pad);
    p.forward_bytes = at;
    at = shared;
    p.lse_at = place(4ull * p.rows_pad);
    p.g_at = place(4ull * p.rows_pad);
    p.d_at = place(2ull * p.rows_pad * p.piece);
    p.rest_at = place(2ull * CE_FINE_ROWS * p.piece);
    // sums of dh: all rows once, or the parts of fewer; those of dW where there are parts
    const auto parts = [](bool small) { return (uint64_t)CE_SPLIT_TILES * (small ? 128 * 128 : 256 * 256); };
    const uint64_t once = ((uint64_t)p.rows_pad + CE_FINE_ROWS) * p.width_pad;
    p.dh_at = place(4 * (once > parts(p.small_products) ? once : parts(p.small_products)));
    p.dw_at = place(p.split_dweight ? 4 * parts(p.small_products) : 0);
    p.dbias_at = place(4ull * (p.rows_pad / ce_dbias_rows(p.small_logits)) * p.vocab_pad);
    p.backward_bytes = at;
    return true;
}

static bool ce_args(const okt_cross_entropy* op, CePlan& p, CeArgs& a) {
    if (!op || !ce_plan(op->rows, op->width, op->vocab, p)) return false;
    if (op->dtype != OKT_BF16 && op->dtype != OKT_F16) return false;
    const auto stride = [&](uint64_t s, uint64_t& to) {
        to = s ? s : op->width;
        return to >= op->width && to <= 1u << 20 && to % 8 == 0;
    };
    if (!stride(op->h_stride, a.h_stride) || !stride(op->weight_stride, a.weight_stride) || !stride(op->dh_stride, a.dh_stride)) return false;
    a.dweight_stride = op->dweight_stride ? op->dweight_stride : op->width;
    if (a.dweight_stride < op->width || a.dweight_stride > 1u << 20 || op->dloss_stride > 1) return false;
    if (op->d_bias && !aligned(op->d_bias, 4)) return false;
    a.rows = (uint32_t)op->rows;
    a.width = op->width;
    a.vocab = op->vocab;
    a.rows_pad = p.rows_pad;
    a.width_pad = p.width_pad;
    a.vocab_pad = p.vocab_pad;
    a.piece = p.piece;
    a.dloss_step = op->dloss_stride;
    a.bias = op->d_bias;
    return true;
}

static void ce_workspace(CeArgs& a, const CePlan& p, char* ws, bool backward) {
    a.header = (CeHeader*)ws;
    a.counts = (float2*)(ws + p.counts_at);
    a.list = (uint32_t*)(ws + p.list_at);
    a.label_of = (int32_t*)(ws + p.label_at);
    a.h = ws + p.h_at;
    a.stats = backward ? nullptr : (float*)(ws + p.stats_at);
    a.said = backward ? nullptr : (float*)(ws + p.said_at);
    a.lse_of = backward ? (float*)(ws + p.lse_at) : nullptr;
    a.g_of = backward ? (float*)(ws + p.g_at) : nullptr;
    a.d = backward ? ws + p.d_at : nullptr;
    a.d_rest = backward ? ws + p.rest_at : nullptr;
    a.dh_sums = backward ? (float*)(ws + p.dh_at) : nullptr;
    a.dw_sums = backward && p.split_dweight ? (float*)(ws + p.dw_at) : nullptr;
    a.dbias_sums = backward ? (float*)(ws + p.dbias_at) : nullptr;
}

// From a tensor's first element to its last one's end.
static size_t ce_extent(uint64_t rows, uint64_t stride, uint32_t width, size_t e) { return rows ? ((rows - 1) * stride + width) * e : 0; }

template <typename T>
static int ce_listed(const CeArgs& a, const void* h, float* loss, const float* lse_in, float* lse_out, const float* dloss, void* dh, hipStream_t s) {
    if (a.rows > CE_DIRECT) {
        hipLaunchKernelGGL(cross_entropy_count_kernel, dim3((a.rows + CE_BLOCK - 1) / CE_BLOCK), dim3(CE_THREADS), 0, s, a, dloss);
        if (const int status = launch_status()) return status;
    }
    const uint32_t rows = (a.rows + CE_GATHERED - 1) / CE_GATHERED, groups = rows < CE_PAD / CE_GATHERED ? CE_PAD / CE_GATHERED : rows;     // the zeros want some, too
    hipLaunchKernelGGL(cross_entropy_gather_kernel<T>, dim3(groups), dim3(CE_THREADS), 0, s, a, (const T*)h, loss, lse_in, lse_out, dloss, (T*)dh);
    return launch_status();
}

// Workgroups of so many tiles of logits: large ones stay on their CU, those of a die with its tiles.
static unsigned ce_logit_groups(const CePlan& p, uint64_t tiles) {
    const uint64_t stay = ce_up(device_cus(), DIES);
    return (unsigned)(p.small_logits || tiles < stay ? tiles : stay);
}

template <class S>
static int ce_join(const CeArgs& a, float* loss, float* lse, hipStream_t s) {
    hipLaunchKernelGGL(cross_entropy_join_kernel, dim3((a.rows + 15) / 16), dim3(CE_JOIN_THREADS), 0, s, a, (a.vocab + S::TILE_M - 1) / S::TILE_M * S::WM, loss, lse);
    return launch_status();
}

template <typename T, class S>
static int ce_forward(const CeArgs& a, const CePlan& p, const void* weight, float* loss, float* lse, hipStream_t s) {
    timing_before(s);
    hipLaunchKernelGGL((cross_entropy_forward_kernel<T, S>), dim3(ce_logit_groups(p, p.logit_groups)), dim3(S::THREADS), 0, s, a, (const T*)weight);
    timing_after(s);
    if (const int status = launch_status()) return status;
    return ce_join<S>(a, loss, lse, s);
}

template <typename T, class S>
static int ce_forward_direct(const CeArgs& a, const CePlan& p, const void* h, const void* weight, float* loss, float* lse, hipStream_t s) {
    timing_before(s);
    hipLaunchKernelGGL((cross_entropy_direct_kernel<T, S>), dim3((unsigned)tile_groups(((a.vocab + S::TILE_M - 1ull) / S::TILE_M) * ((a.rows + S::TILE_N - 1ull) / S::TILE_N))), dim3(S::THREADS), 0, s, a, (const T*)h, (const T*)weight, loss, lse);
    timing_after(s);
    if (const int status = launch_status()) return status;
    return ce_join<S>(a, loss, lse, s);
}

// Tiles of 64 columns for 128 where that leaves no CU with two (125 x 776 x 10007, 157 of them: 16.2 -> 15.2 us; 3 x 880 x 18612, 291: 16.3 -> 19.8;
// gradient of 1000 x 2048 x 500, 64 of them: 48.1 -> 45.7, of 300 x 4096 x 5000 100.8 -> 96.5).
static uint64_t ce_thin_tiles(uint64_t columns, uint64_t rows) {
    return (columns + Thin::TILE_M - 1) / Thin::TILE_M * (rows ? (rows + Thin::TILE_N - 1) / Thin::TILE_N : 1);
}
static bool ce_thin(uint64_t columns, uint64_t rows) { return ce_thin_tiles(columns, rows) <= device_cus(); }

struct CeGradients { void *dh, *dweight; float* dbias; };

template <typename T, typename W, class S>
static int ce_products(const CeArgs& a, const CePlan& p, const void* weight, const CeGradients& g, uint32_t from, uint32_t columns, hipStream_t s) {
    const uint32_t dh_groups = g.dh ? (uint32_t)p.dh_groups : 0, dw_groups = g.dweight ? (uint32_t)p.dweight_groups : 0;
    // one launch where dh's tiles do not fill the chip by themselves (8192 x 4096 x 128000: two 19.8 ms, one 20.2; 22 x 752 x 112: two 31 us, one 25)
    const auto launch = [&](uint32_t dh, uint32_t dw) {              // workgroups of each
        if (dh + dw == 0) return (int)OKT_OK;
        hipLaunchKernelGGL((cross_entropy_products_kernel<T, W, S>), dim3(dh + dw), dim3(S::THREADS), 0, s, a, (const T*)weight, (W*)g.dweight, from, columns, dh);
        return launch_status();
    };
    const bool apart = dh_groups > CE_SPLIT_TILES;
    if (const int status = launch(dh_groups, apart ? 0 : dw_groups)) return status;
    if (apart)
        if (const int status = launch(0, dw_groups)) return status;
    const bool last = from + (uint64_t)columns >= a.vocab;
    const uint64_t tiles = (uint64_t)((a.width_pad + S::TILE_M - 1) / S::TILE_M) * ((columns + S::TILE_N - 1) / S::TILE_N);
    const uint32_t across = (a.width + WAVE * 8 - 1) / (WAVE * 8);
    const auto rows = [&](uint32_t n) {                              // workgroups of so many rows, at most 2^16 times `across`
        const uint32_t blocks = (n + CE_THREADS / WAVE - 1) / (CE_THREADS / WAVE);
        return (blocks < 1u << 16 ? blocks : 1u << 16) * across;
    };
    const CeFinish f = {g.dh && last ? rows(a.rows) : 0, g.dweight && p.split_dweight && tiles * 2 <= CE_SPLIT_TILES ? rows(columns) : 0};
    const uint32_t bias = g.dbias && last ? (a.vocab + CE_THREADS - 1) / CE_THREADS : 0;
    if (f.dh_groups + f.dw_groups + bias == 0) return OKT_OK;
    hipLaunchKernelGGL((cross_entropy_finish_kernel<T, W, S>), dim3(f.dh_groups + f.dw_groups + bias), dim3(CE_THREADS), 0, s, a, (T*)g.dh,
                       (W*)g.dweight, g.dbias, from, columns, f);
    return launch_status();
}

template <typename T, typename W>
static int ce_backward(CeArgs a, const CePlan& p, const void* weight, CeGradients g, hipStream_t s) {
    if (a.rows == 0) g.dh = nullptr;
    static_assert(Thin::TILE_N == Spread::TILE_N && Thin::WN == Spread::WN, "");
    a.logit_tile_n = p.small_logits ? Spread::TILE_N : Large::TILE_N;
    a.logit_parts_n = p.small_logits ? Spread::WN : Large::WN;
    for (uint64_t from = 0; from < a.vocab; from += p.piece) {
        const uint32_t first = (uint32_t)from, columns = a.vocab - first < p.piece ? a.vocab - first : p.piece;
        const dim3 groups(ce_logit_groups(p, p.piece_groups));
        timing_before(s);
        if (p.small_logits && ce_thin(columns, a.rows))
            hipLaunchKernelGGL((cross_entropy_gradient_kernel<T, Thin>), dim3((unsigned)tile_groups(ce_thin_tiles(columns, a.rows))), dim3(Thin::THREADS), 0, s, a,
                               (const T*)weight, first, columns);
        else if (p.small_logits)
            hipLaunchKernelGGL((cross_entropy_gradient_kernel<T, Spread>), groups, dim3(Spread::THREADS), 0, s, a, (const T*)weight, first, columns);
        else
            hipLaunchKernelGGL((cross_entropy_gradient_kernel<T, Large>), groups, dim3(Large::THREADS), 0, s, a, (const T*)weight, first, columns);
        timing_after(s);
        if (const int status = launch_status()) return status;
        const auto products = p.narrow_products ? ce_products<T, W, Narrow> : p.small_products ? ce_products<T, W, Small> : ce_products<T, W, Large>;
        if (const int status = products(a, p, weight, g, first, columns, s)) return status;
    }
    return OKT_OK;
}

// Whether every workgroup of the logits can list the rows by itself, and reach them all from the first one.
static bool ce_direct(const CeArgs& a, const CePlan& p) {
    return p.small_logits && a.rows <= CE_DIRECT && ce_extent(a.rows, a.h_stride, a.width, 2) < 1ull << 31;
}

template <typename T>
static int ce_run_forward(const CeArgs& a, const CePlan& p, const void* h, const void* weight, float* loss, float* lse, hipStream_t s) {
    if (ce_direct(a, p)) return ce_thin(a.vocab, a.rows) ? ce_forward_direct<T, Thin>(a, p, h, weight, loss, lse, s) : ce_forward_direct<T, Spread>(a, p, h, weight, loss, lse, s);
    if (const int status = ce_listed<T>(a, h, loss, nullptr, lse, nullptr, nullptr, s)) return status;
    return p.small_logits ? ce_forward<T, Spread>(a, p, weight, loss, lse, s) : ce_forward<T, Large>(a, p, weight, loss, lse, s);
}
template <typename T>
static int ce_run_backward(const CeArgs& a, const CePlan& p, const void* h, const void* weight, const float* lse, const float* dloss, const CeGradients& g, bool wide,
                           hipStream_t s) {
    if (const int status = ce_listed<T>(a, h, nullptr, lse, nullptr, dloss, g.dh, s)) return status;
    return wide ? ce_backward<T, float>(a, p, weight, g, s) : ce_backward<T, T>(a, p, weight, g, s);
}

}  // namespace okt

extern "C" {

size_t okt_cross_entropy_workspace_bytes(uint64_t rows, uint32_t width, uint32_t vocab) {
    okt::CePlan p;
    if (!okt::ce_plan(rows, width, vocab, p)) return 0;
    return p.forward_bytes > p.backward_bytes ? p.forward_bytes : p.backward_bytes;
}

int okt_cross_entropy_forward(const okt_cross_entropy* op, const void* d_h, const void* d_weight, const int64_t* d_labels, float* d_loss_out,
                              float* d_lse_out, void* d_ws, size_t ws_bytes, void* stream) {
    using namespace okt;
    CePlan p;
    CeArgs a;
    if (!ce_args(op, p, a)) return OKT_ERR_INVALID_ARG;
    if (a.rows == 0) return OKT_OK;
    if (!d_h || !d_weight || !d_labels || !d_loss_out || !aligned(d_h, 16) || !aligned(d_weight, 16) || !aligned(d_labels, 8) ||
        !aligned(d_loss_out, 4) || !aligned(d_lse_out, 4)) return OKT_ERR_INVALID_ARG;
    const struct { const void* p; size_t bytes; } in[] = {{d_h, ce_extent(a.rows, a.h_stride, a.width, 2)},
                                                          {d_weight, ce_extent(a.vocab, a.weight_stride, a.width, 2)},
                                                          {d_labels, 8ull * a.rows}, {a.bias, a.bias ? 4ull * a.vocab : 0}};
    for (const auto& t : in)
        for (const float* out : {d_loss_out, d_lse_out})
            if (out && t.bytes && overlap(out, 4ull * a.rows, t.p, t.bytes)) return OKT_ERR_INVALID_ARG;
    if (d_lse_out && overlap(d_loss_out, 4ull * a.rows, d_lse_out, 4ull * a.rows)) return OKT_ERR_INVALID_ARG;
    if (!d_ws || !aligned(d_ws, 256) || ws_bytes < p.forward_bytes) return OKT_ERR_WORKSPACE;
    a.labels = d_labels;
    ce_workspace(a, p, (char*)d_ws, false);
    const hipStream_t s = (hipStream_t)stream;
    return op->dtype == OKT_BF16 ? ce_run_forward<__bf16>(a, p, d_h, d_weight, d_loss_out, d_lse_out, s)
                                 : ce_run_forward<_Float16>(a, p, d_h, d_weight, d_loss_out, d_lse_out, s);
}

int okt_cross_entropy_backward(const okt_cross_entropy* op, const void* d_h, const void* d_weight, const int64_t* d_labels, const float* d_lse,
                               const float* d_dloss, void* d_dh_out, void* d_dweight_out, float* d_dbias_out, void* d_ws, size_t ws_bytes, void* stream) {
    using namespace okt;
    CePlan p;
    CeArgs a;
    if (!ce_args(op, p, a)) return OKT_ERR_INVALID_ARG;
    const bool wide = op->dweight_dtype == OKT_F32;
    if (!wide && op->dweight_dtype != op->dtype) return OKT_ERR_INVALID_ARG;
    if (!wide && a.dweight_stride % 8 != 0) return OKT_ERR_INVALID_ARG;
    if ((d_dbias_out && !a.bias) || (!d_dh_out && !d_dweight_out && !d_dbias_out)) return OKT_ERR_INVALID_ARG;
    if (!aligned(d_dweight_out, wide ? 4 : 16) || !aligned(d_dbias_out, 4) || !aligned(d_dh_out, 16)) return OKT_ERR_INVALID_ARG;
    if (!d_weight || !aligned(d_weight, 16)) return OKT_ERR_INVALID_ARG;
    if (a.rows && (!d_h || !d_labels || !d_lse || !d_dloss || !aligned(d_h, 16) || !aligned(d_labels, 8) || !aligned(d_lse, 4) || !aligned(d_dloss, 4)))
        return OKT_ERR_INVALID_ARG;
    const size_t scalars = 4ull * (a.rows ? (a.rows - 1ull) * a.dloss_step + 1 : 0);
    const struct { const void* p; size_t bytes; } t[] = {
        {d_dh_out, ce_extent(a.rows, a.dh_stride, a.width, 2)}, {d_dweight_out, ce_extent(a.vocab, a.dweight_stride, a.width, wide ? 4 : 2)},
        {d_dbias_out, 4ull * a.vocab}, {d_h, ce_extent(a.rows, a.h_stride, a.width, 2)}, {d_weight, ce_extent(a.vocab, a.weight_stride, a.width, 2)},
        {d_labels, 8ull * a.rows}, {d_lse, 4ull * a.rows}, {d_dloss, scalars}, {a.bias, 4ull * a.vocab}};
    for (int out = 0; out < 3; ++out)
        for (int other = out + 1; other < 9; ++other)
            if (t[out].p && t[other].p && t[out].bytes && t[other].bytes && overlap(t[out].p, t[out].bytes, t[other].p, t[other].bytes)) return OKT_ERR_INVALID_ARG;
    if (!d_ws || !aligned(d_ws, 256) || ws_bytes < p.backward_bytes) return OKT_ERR_WORKSPACE;
    a.labels = d_labels;
    ce_workspace(a, p, (char*)d_ws, true);
    if (!d_dbias_out) a.dbias_sums = nullptr;
    const hipStream_t s = (hipStream_t)stream;
    const CeGradients g = {d_dh_out, d_dweight_out, d_dbias_out};
    return op->dtype == OKT_BF16 ? ce_run_backward<__bf16>(a, p, d_h, d_weight, d_lse, d_dloss, g, wide, s)
                                 : ce_run_backward<_Float16>(a, p, d_h, d_weight, d_lse, d_dloss, g, wide, s);
}

}  // extern "C"
