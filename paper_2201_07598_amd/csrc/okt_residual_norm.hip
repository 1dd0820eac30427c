// okt_residual_norm_forward / _backward: what stands between two blocks of a layer, in one
// pass over the rows.
//
//   a = Npost(u) or u        the norm after the block
//   h = alpha x + g drop(a)  dropout, gate and the scaled residual stream
//   y = Npre(h)              the norm before the next block
//
// with N(v) = (v - m) r w + b, m = mean (0 for RMS), r = 1 / sqrt(mean (v - m)^2 + eps).
// Backward, with w' = dout w and xhat = (v - m) r:
//   dv = r (w' - mean w' - xhat mean(w' xhat))     (RMS: without mean w')
//   dw = sum over rows of dout xhat,  db = sum of dout,  dg = sum of dh drop(a)
//
// A row lives in the registers of a wave or of a workgroup (Layout: groups of eight columns a
// thread), so the mean, the centred squares and the result are taken from one read
// of it; everything is fp32 between the load and the one rounding of the store.  The second norm reads h as it was
// stored, since that is what the backward pass has.  The mask of the dropout is drawn
// again in the backward pass: a group of eight columns is a block of the random field.
// Workgroups walk over the rows and keep the parameters, and backward the sums over rows, in
// registers; those sums leave as one partial row per workgroup, which a second launch
// adds in a fixed order (no atomics: the result does not change from run to run).
// Bound by memory: forward 4 elements a place, backward 5 or 6.  From call to call:
//   forward   16384 x 1024 bf16   29 us, 4.6 TB/s of 134 MB (the kernel 25)
//             128 x 768 fp32      8-10 us, 8.0 of which are the host's; the kernel 4.8
//             16384 x 1024 bf16, both norms, 32 gates and dropout 41 us; RMS, one gate, no dropout 34.5
//   backward  16384 x 1024 bf16   38 us, 4.4 TB/s of 168 MB (the kernel 28, the add 4 and the step between them)
//             4099 x 2500 fp16, both norms and a gate
//                                 52 us, 2.4 TB/s of 123 MB (the kernel 45, the add 6).  Of that 17 us are
//             there with one row a workgroup, too: two launches, the parameters on the way in, their
//             gradients on the way out; and rows of 5000 bytes begin and end inside a line of the
//             caches (16384 rows of 2500 133-140 us, of 2504 120).  16384 x 768 50, 16384 x 1024 55, 8192 x 4096 99,
//             2048 x 8192 71 (no biases): rows of two groups a thread, one workgroup a CU, whose sums are in LDS
#include "okt_element.h"
#include "okt_random.h"

namespace okt {

// ------------------------------------------------------------------ sizes (host)

constexpr uint32_t NORM_MIN_WIDTH = 8, NORM_MAX_WIDTH = 8192;
constexpr uint64_t NORM_MAX_ROWS = 1ull << 40;
constexpr uint32_t NORM_BACKWARD_GROUPS = 512;     // workgroups aimed at: two to a CU
constexpr uint32_t NORM_SUMS = 5;                  // pre w, pre b, post w, post b, gate

// Threads that hold a row, eight columns each `vecs` times over.  One wave where it can: its
// sums need no barrier, and four rows of four waves are on their way together (backward, 16384 rows:
// of 1024 39 us against 49 at one group and two waves, of 768 31 against 49).  With a norm after
// the block or a gate the kernel holds twice the sums and ends with as many more of them to add over its waves,
// which only many rows are worth: with both, of 1024 and 16-bit, 16384 rows 55 against 67 us, 8192 35 against 38,
// 4096 30 against 26; of fp32, where the registers go to fetched rows, 16384 rows 94 against 89.
struct NormShape { uint32_t lanes, vecs; };

static NormShape norm_shape(uint32_t width, uint64_t rows, int dtype, bool backward_of_all) {
    if (width <= 512) return {WAVE, 1};
    if (width <= 1024 && (!backward_of_all || (dtype != OKT_F32 && rows >= 8192))) return {WAVE, 2};
    if (width <= 4096) return {(width + WAVE * 8 - 1) / (WAVE * 8) * WAVE, 1};
    return {512, 2};
}

static uint32_t rows_at_once(NormShape s) { return s.lanes == WAVE ? 4 : 1; }

// How the backward pass deals out the rows of gates.  A workgroup owns `chunk` rows that either are
// whole gates' rows (parts == 1: it writes their dgate itself) or lie within one gate
// (parts workgroups to a gate, whose partial sums the second launch adds).
struct NormPlan { uint64_t chunk, rows_per_gate, gates, groups; uint32_t parts; };

static NormPlan norm_plan(uint64_t rows, uint64_t rows_per_gate, uint32_t at_once) {
    NormPlan p;
    p.rows_per_gate = rows_per_gate == 0 || rows_per_gate > rows ? rows : rows_per_gate;
    if (rows == 0) return {1, 1, 1, 0, 0};             // sums over nothing
    p.gates = (rows + p.rows_per_gate - 1) / p.rows_per_gate;
    p.chunk = (rows + NORM_BACKWARD_GROUPS - 1) / NORM_BACKWARD_GROUPS;
    p.chunk = (p.chunk + at_once - 1) / at_once * at_once;
    if (p.rows_per_gate <= p.chunk) {
        p.chunk = (p.chunk + p.rows_per_gate - 1) / p.rows_per_gate * p.rows_per_gate;
        p.parts = 1;
        p.groups = (rows + p.chunk - 1) / p.chunk;
    } else {
        p.parts = (uint32_t)((p.rows_per_gate + p.chunk - 1) / p.chunk);
        p.chunk = (p.rows_per_gate + p.parts - 1) / p.parts;
        p.groups = p.gates * p.parts;
    }
    return p;
}

static size_t norm_ws_bytes(uint64_t rows, uint32_t width, uint64_t rows_per_gate) {
    uint64_t groups = 0;
    for (uint32_t at_once : {1u, 4u}) {
        const uint64_t n = norm_plan(rows, rows_per_gate, at_once).groups;
        groups = n > groups ? n : groups;
    }
    return (size_t)(NORM_SUMS * groups * width * sizeof(float) + 255) & ~(size_t)255;
}

// ------------------------------------------------------------------ device

struct NormArgs {
    uint64_t rows, rows_per_gate;
    uint32_t width, site;
    float eps, alpha, inv_width;
    bool layer;
    DropoutRule drop;                               // bar 65536: none
    const uint64_t* seed;
    const float *post_w, *post_b, *gate, *pre_w, *pre_b;
    uint64_t u_stride, x_stride, h_stride, y_stride, dh_stride, dy_stride, dx_stride, du_stride;
    float4* stats;
    // backward
    uint64_t chunk, groups;
    uint32_t parts;
    float* partial;                                 // [NORM_SUMS][groups][width]
    float* dgate;
};

// Sum over the wave, the same in every lane, in the vector unit alone.
__device__ __forceinline__ float wave_sum_f32(float v) {
#define OKT_DPP_ADD(ctrl, rows) \
    v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, rows, 0xf, false))
    OKT_DPP_ADD(0xB1, 0xf);                         // neighbours
    OKT_DPP_ADD(0x4E, 0xf);                         // pairs of a quad
    OKT_DPP_ADD(0x141, 0xf);                        // quads of half a row
    OKT_DPP_ADD(0x140, 0xf);                        // halves of a row of 16
    OKT_DPP_ADD(0x142, 0xa);                        // row 0 into 1, 2 into 3
    OKT_DPP_ADD(0x143, 0xc);                        // rows 0-1 into 2-3
#undef OKT_DPP_ADD
    return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Clears the slots of row_sums, before its first call.
template <typename L>
__device__ __forceinline__ void clear_slots(float2* slots) {
    if (!L::one) {
        if (threadIdx.x < L::slots) slots[threadIdx.x] = make_float2(0.0f, 0.0f);
        __syncthreads();
    }
}

// How a kernel holds rows: ONE wave each, or a workgroup of up to THREADS each; VECS groups
// of eight columns a thread.
template <bool ONE, int VECS, int THREADS>
struct Layout {
    static constexpr bool one = ONE;
    static constexpr int vecs = VECS, threads = THREADS, slots = 2 * THREADS / WAVE;
    };

// Two sums over the threads of a row.  `turn` alternates between two sets of slots, so one
// barrier a call is enough: a set is written again only after the next call's barrier.
template <typename L>
__device__ __forceinline__ void row_sums(float& a, float& b, float2* slots, int& turn) {
    a = wave_sum_f32(a);
    b = wave_sum_f32(b);
    if (!L::one) {
        float2* s = slots + turn * (L::threads / WAVE);
        if (threadIdx.x % WAVE == 0) s[threadIdx.x / WAVE] = make_float2(a, b);
        __syncthreads();
        a = b = 0.0f;
#pragma unroll
        for (int w = 0; w < L::threads / WAVE; ++w) {          // slots of waves there are not hold 0
            a += s[w].x;
            b += s[w].y;
        }
        turn ^= 1;
    }
}

__device__ __forceinline__ float sum_eight(f32x8 v) {
    return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// The columns of one thread: groups of eight, as many apart as threads hold the row.  A
// group that the row ends in, or before, is read as the last eight elements of the row and moved into
// place, so every load of a row is one wide load that depends on nothing.  What it reads of another
// thread's columns is dropped, so an output may take an input's place.
template <typename L>
struct Columns {
    uint32_t lane, lanes, width, at[L::vecs], skip[L::vecs];
    __device__ __forceinline__ Columns(uint32_t lane_, uint32_t lanes_, uint32_t width_) : lane(lane_), lanes(lanes_), width(width_) {
#pragma unroll
        for (int v = 0; v < L::vecs; ++v) {
            const uint32_t col = group(v) * 8 < width ? group(v) * 8 : width;
            at[v] = col + 8 <= width ? col : width - 8;
            skip[v] = col - at[v];                                  // 8: no columns
        }
    }
    __device__ __forceinline__ uint32_t group(int v) const { return v * lanes + lane; }
    __device__ __forceinline__ uint32_t first(int v) const { return at[v] + skip[v]; }
    __device__ __forceinline__ int count(int v) const { return 8 - (int)skip[v]; }

    template <typename T>
    struct Raw { typename Eight<T>::vec v[L::vecs]; };

    template <typename T>
    __device__ __forceinline__ Raw<T> fetch(const T* row) const {
        Raw<T> r;
#pragma unroll
        for (int v = 0; v < L::vecs; ++v) r.v[v] = raw_eight(row + at[v]);
        return r;
    }
    template <typename T>
    __device__ __forceinline__ void open(f32x8 (&to)[L::vecs], Raw<T> r) const {
#pragma unroll
        for (int v = 0; v < L::vecs; ++v) {
            if (skip[v] - 1u < 7u) r.v[v] = skip_elements<T>(r.v[v], skip[v]);
            to[v] = skip[v] < 8 ? __builtin_convertvector(r.v[v], f32x8) : 0.0f;
        }
    }
    template <typename T>
    __device__ __forceinline__ void load(f32x8 (&to)[L::vecs], const T* row) const { open<T>(to, fetch<T>(row)); }

    template <typename T>
    __device__ __forceinline__ void store(T* row, const f32x8 (&from)[L::vecs]) const {
#pragma unroll
        for (int v = 0; v < L::vecs; ++v) {
            T* p = row + first(v);
            if (!skip[v]) store_eight(p, from[v]);
            else if (skip[v] < 8) store_some(p, from[v], 8 - (int)skip[v]);
        }
    }
};

// Mean and reciprocal deviation of a row: the mean first, then the centred squares.
template <typename L>
__device__ __forceinline__ float2 row_statistics(const f32x8 (&v)[L::vecs], const Columns<L>& cols, const NormArgs& a,
                                                 float2* slots, int& turn) {
    float mean = 0.0f, none = 0.0f, squares = 0.0f;
    if (a.layer) {
#pragma unroll
        for (int i = 0; i < L::vecs; ++i) mean += sum_eight(v[i]);      // columns past the width hold 0
        row_sums<L>(mean, none, slots, turn);
        mean *= a.inv_width;
    }
#pragma unroll
    for (int i = 0; i < L::vecs; ++i) {
        const int n = cols.count(i);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float d = j < n ? v[i][j] - mean : 0.0f;
            squares = __builtin_fmaf(d, d, squares);
        }
    }
    none = 0.0f;
    row_sums<L>(squares, none, slots, turn);
    return make_float2(mean, 1.0f / __builtin_sqrtf(__builtin_fmaf(squares, a.inv_width, a.eps)));
}

// Multiplies by scale what the random field keeps and clears the rest.
template <typename L>
__device__ __forceinline__ void drop_row(f32x8 (&v)[L::vecs], const Columns<L>& cols, uint64_t row, RandomKey key,
                                         const NormArgs& a) {
#pragma unroll
    for (int i = 0; i < L::vecs; ++i) {
        const RandomBlock b = random_block(key, cols.first(i) / 8, (uint32_t)row, (uint32_t)(row >> 32), a.site);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i][j] = kept(b, j, a.drop.bar) ? v[i][j] * a.drop.scale : 0.0f;
    }
}

template <typename T, typename L>
__global__ __launch_bounds__(L::threads) void norm_forward_kernel(NormArgs a, const T* u, const T* x, T* h,
                                                                                   T* y) {
    constexpr int AT_ONCE = L::one ? L::threads / WAVE : 1;
    __shared__ float2 slots[L::slots];
    clear_slots<L>(slots);
    int turn = 0;
    const Columns<L> cols(L::one ? threadIdx.x % WAVE : threadIdx.x, L::one ? WAVE : blockDim.x, a.width);
    const bool drops = a.drop.bar != 65536u;
    RandomKey key = {0, 0};
    if (drops) key = random_key(a.seed);
    f32x8 pre_w[L::vecs], pre_b[L::vecs];
    if (a.pre_w) cols.load(pre_w, a.pre_w);
    if (a.pre_b) cols.load(pre_b, a.pre_b);
    for (uint64_t row = (uint64_t)blockIdx.x * AT_ONCE + (L::one ? threadIdx.x / WAVE : 0); row < a.rows;
         row += (uint64_t)gridDim.x * AT_ONCE) {
        f32x8 s[L::vecs], r[L::vecs];
        float4 st = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        cols.load(s, u + row * a.u_stride);
        cols.load(r, x + row * a.x_stride);
        if (a.post_w) {
            const float2 m = row_statistics<L>(s, cols, a, slots, turn);
            st.x = m.x;
            st.y = m.y;
            f32x8 w[L::vecs];
            cols.load(w, a.post_w);
#pragma unroll
            for (int i = 0; i < L::vecs; ++i) s[i] = (s[i] - m.x) * m.y * w[i];
            if (a.post_b) {
                cols.load(w, a.post_b);
#pragma unroll
                for (int i = 0; i < L::vecs; ++i) s[i] += w[i];
            }
        }
        if (drops) drop_row<L>(s, cols, row, key, a);
        if (a.gate) {
            f32x8 g[L::vecs];
            cols.load(g, a.gate + row / a.rows_per_gate * a.width);
#pragma unroll
            for (int i = 0; i < L::vecs; ++i) s[i] *= g[i];
        }
#pragma unroll
        for (int i = 0; i < L::vecs; ++i) s[i] = __builtin_convertvector(
            __builtin_convertvector(a.alpha * r[i] + s[i], typename Eight<T>::vec), f32x8);
        if (h) cols.store(h + row * a.h_stride, s);
        if (a.pre_w) {
            const float2 m = row_statistics<L>(s, cols, a, slots, turn);
            st.z = m.x;
            st.w = m.y;
#pragma unroll
            for (int i = 0; i < L::vecs; ++i) s[i] = (s[i] - m.x) * m.y * pre_w[i];
            if (a.pre_b) {
#pragma unroll
                for (int i = 0; i < L::vecs; ++i) s[i] += pre_b[i];
            }
            cols.store(y + row * a.y_stride, s);
        }
        if (a.stats && cols.lane == 0) a.stats[row] = st;
    }
}

// A sum over rows for each column of a thread: in registers, or in LDS.
template <typename L, bool LDS>
struct ColumnSums {
    f32x8 r[LDS ? 1 : L::vecs];
    float* at;                                          // this thread's eight columns of the first group
    __device__ __forceinline__ explicit ColumnSums(float* shared) : at(shared + threadIdx.x * 8) { clear(); }
    __device__ __forceinline__ void clear() {
#pragma unroll
        for (int i = 0; i < L::vecs; ++i) {
            if (LDS) *reinterpret_cast<f32x8*>(at + i * L::threads * 8) = 0.0f;
            else r[LDS ? 0 : i] = 0.0f;
        }
    }
    __device__ __forceinline__ void add(int i, f32x8 v) {
        if (LDS) *reinterpret_cast<f32x8*>(at + i * L::threads * 8) += v;
        else r[LDS ? 0 : i] += v;
    }
    __device__ __forceinline__ void add(int i, f32x8 a, f32x8 b) {          // a b, without rounding the product
        f32x8 sum = LDS ? *reinterpret_cast<f32x8*>(at + i * L::threads * 8) : r[LDS ? 0 : i];
        sum = __builtin_elementwise_fma(a, b, sum);
        if (LDS) *reinterpret_cast<f32x8*>(at + i * L::threads * 8) = sum;
        else r[LDS ? 0 : i] = sum;
    }
    __device__ __forceinline__ void get(f32x8 (&to)[L::vecs]) const {
#pragma unroll
        for (int i = 0; i < L::vecs; ++i) to[i] = LDS ? *reinterpret_cast<const f32x8*>(at + i * L::threads * 8) : r[LDS ? 0 : i];
    }
};

// The gradient of a norm's input from the gradient of its output (in place), and what this
// row adds to the gradients of its weight and bias.
template <typename L, bool BIAS, typename W, typename B>
__device__ __forceinline__ void norm_input_gradient(f32x8 (&d)[L::vecs], const f32x8 (&v)[L::vecs], const f32x8 (&w)[L::vecs],
                                                    float mean, float r, W& dw, B& db, const NormArgs& a, float2* slots, int& turn) {
    float plain = 0.0f, along = 0.0f;
    f32x8 xhat[L::vecs];
#pragma unroll
    for (int i = 0; i < L::vecs; ++i) {
        xhat[i] = (v[i] - mean) * r;
        dw.add(i, d[i], xhat[i]);
        if (BIAS) db.add(i, d[i]);
        d[i] *= w[i];
        plain += sum_eight(d[i]);
#pragma unroll
        for (int j = 0; j < 8; ++j) along = __builtin_fmaf(d[i][j], xhat[i][j], along);
    }
    row_sums<L>(plain, along, slots, turn);
    plain = a.layer ? plain * a.inv_width : 0.0f;
    along *= a.inv_width;
#pragma unroll
    for (int i = 0; i < L::vecs; ++i) d[i] = __builtin_elementwise_fma(xhat[i], (f32x8)-along, d[i] - plain) * r;
}

// Adds what the waves of a workgroup that work on different rows hold, and writes it out.
template <typename L, typename S>
__device__ __forceinline__ void put_sums(const S& sums, const Columns<L>& cols, float* to, float* shared) {
    f32x8 v[L::vecs];
    sums.get(v);
    if (L::one) {
        constexpr int SPAN = WAVE * L::vecs * 8;
        const int wave = threadIdx.x / WAVE;
        __syncthreads();
#pragma unroll
        for (int i = 0; i < L::vecs; ++i) *reinterpret_cast<f32x8*>(shared + wave * SPAN + cols.group(i) * 8) = v[i];
        __syncthreads();
        for (uint32_t c = threadIdx.x; c < cols.width; c += 256)
            to[c] = (shared[c] + shared[SPAN + c]) + (shared[2 * SPAN + c] + shared[3 * SPAN + c]);
    } else {
        cols.store(to, v);
    }
}

// ALL: with a norm after the block or a gate; BIAS: a norm has one.  Without, the registers
// they take are free.  DROP (of ALL): something may be dropped.
template <typename T, typename L, bool ALL, bool BIAS, bool DROP>
__global__ __launch_bounds__(L::threads) void norm_backward_kernel(
    NormArgs a, const T* u, const T* h, const T* dh, const T* dy, T* dx, T* du) {
    constexpr int AT_ONCE = L::one ? L::threads / WAVE : 1;
    __shared__ float2 slots[L::slots];
    clear_slots<L>(slots);
    // rows of two groups a thread: as many sums as LDS holds lie there (2048 rows of 8192 with both norms
    // and their biases, fp16: 83 us, all in registers 414), and in fp32, where registers are short all the same, no
    // row is fetched ahead (132 us, ahead 195; fp16 83, not ahead 90)
    constexpr int SPAN = L::threads * L::vecs * 8, LDS_SUMS = ALL && !L::one && L::vecs == 2 ? 32768 / SPAN : 0;
    constexpr bool AHEAD = L::one || L::vecs == 1 || sizeof(T) == 2;
    __shared__ __attribute__((aligned(32))) float shared[L::one ? SPAN : LDS_SUMS ? LDS_SUMS * SPAN : 8];
    int turn = 0;
    const Columns<L> cols(L::one ? threadIdx.x % WAVE : threadIdx.x, L::one ? WAVE : blockDim.x, a.width);
    const bool drops = a.drop.bar != 65536u;
    RandomKey key = {0, 0};
    if (drops) key = random_key(a.seed);
    f32x8 pre_w[L::vecs], post_w[L::vecs], post_b[L::vecs];
    ColumnSums<L, (LDS_SUMS > 0)> dpost_w(shared);
    ColumnSums<L, (LDS_SUMS > 1)> dgate(shared + (LDS_SUMS > 1 ? SPAN : 0));
    ColumnSums<L, (LDS_SUMS > 2)> dpre_w(shared + (LDS_SUMS > 2 ? 2 * SPAN : 0));
    ColumnSums<L, (LDS_SUMS > 3 && BIAS)> dpost_b(shared + (LDS_SUMS > 3 ? 3 * SPAN : 0));
    ColumnSums<L, false> dpre_b(shared);
    if (a.pre_w) cols.load(pre_w, a.pre_w);
    if (ALL && a.post_w) cols.load(post_w, a.post_w);
    if (ALL && BIAS && a.post_b) cols.load(post_b, a.post_b);

    // Without a gate the rows are dealt in turn, so that what the workgroups read at a time lies
    // together (65536 rows of 768 110.0 -> 96.8 us, 8192 of 4096 79.2 -> 73.0); the kernel with gates, whose rows
    // take longer than their loads, has nothing from it (16384 rows of 2560 119.5 -> 121.5).
    const uint64_t gate0 = !ALL ? 0 : a.parts > 1 ? blockIdx.x / a.parts : blockIdx.x * (a.chunk / a.rows_per_gate);
    uint64_t begin = a.parts > 1 ? gate0 * a.rows_per_gate + blockIdx.x % a.parts * a.chunk : blockIdx.x * a.chunk;
    uint64_t last = begin + a.chunk;
    if (a.parts > 1 && last > (gate0 + 1) * a.rows_per_gate) last = (gate0 + 1) * a.rows_per_gate;
    if (!ALL) begin = blockIdx.x * AT_ONCE;
    if (!ALL || last > a.rows) last = a.rows;
    const uint32_t step = ALL ? AT_ONCE : gridDim.x * AT_ONCE;

    // A row's loads are issued before the row ahead of it is worked on.
    typename Columns<L>::template Raw<T> next_dh, next_u, next_h, next_dy;
    float4 next_st;
    const auto fetch = [&](uint64_t row) {
        next_st = a.stats[row];
        if (dh) next_dh = cols.fetch(dh + row * a.dh_stride);
        if (ALL) next_u = cols.fetch(u + row * a.u_stride);
        if (a.pre_w) {
            next_h = cols.fetch(h + row * a.h_stride);
            next_dy = cols.fetch(dy + row * a.dy_stride);
        }
    };
    for (uint64_t gate = gate0; begin < last || gate == gate0; ++gate) {
        // the rows of one gate; a workgroup whose part of it is empty passes through once
        uint64_t end = (gate + 1) * a.rows_per_gate;
        if (!ALL || end > last) end = last;
        f32x8 g[L::vecs];
        if (ALL && a.gate) cols.load(g, a.gate + gate * a.width);
        uint64_t row = begin + (L::one ? threadIdx.x / WAVE : 0);
        if (AHEAD && row < end) fetch(row);
        for (; row < end; row += step) {
            if (!AHEAD) fetch(row);
            const float4 st = next_st;
            f32x8 d[L::vecs], v[L::vecs], o[L::vecs], su[L::vecs];
#pragma unroll
            for (int i = 0; i < L::vecs; ++i) d[i] = 0.0f;
            if (dh) cols.template open<T>(d, next_dh);
            if (ALL) cols.template open<T>(su, next_u);
            if (a.pre_w) {
                cols.template open<T>(v, next_h);
                cols.template open<T>(o, next_dy);
            }
            if (AHEAD && row + step < end) fetch(row + step);
            if (a.pre_w) {
                norm_input_gradient<L, BIAS>(o, v, pre_w, st.z, st.w, dpre_w, dpre_b, a, slots, turn);
#pragma unroll
                for (int i = 0; i < L::vecs; ++i) d[i] += o[i];
            }
#pragma unroll
            for (int i = 0; i < L::vecs; ++i) v[i] = a.alpha * d[i];
            cols.store(dx + row * a.dx_stride, v);
            if (drops) drop_row<L>(d, cols, row, key, a);
            if (ALL) {
                if (a.gate) {
#pragma unroll
                    for (int i = 0; i < L::vecs; ++i) {
                        f32x8 s = su[i];
                        if (a.post_w) s = (s - st.x) * st.y * post_w[i];
                        if (BIAS && a.post_b) s += post_b[i];
                        // d holds the mask and its scale already.  Where it is 0, as at every place that is
                        // dropped, the place adds 0: 0 times a value that is not finite would stay in the gate's sum.
                        // (A branch, and the mask's own words, take 7 to 12 registers more, with which a CU holds one
                        // workgroup of 4099 x 2500 where it holds two; so it costs 1 us of 57.)
                        if (DROP) {
#pragma unroll
                            for (int j = 0; j < 8; ++j) s[j] = d[i][j] != 0.0f ? s[j] : 0.0f;
                        }
                        dgate.add(i, d[i], s);
                        d[i] *= g[i];
                    }
                }
                if (a.post_w) norm_input_gradient<L, BIAS>(d, su, post_w, st.x, st.y, dpost_w, dpost_b, a, slots, turn);
            }
            cols.store(du + row * a.du_stride, d);
        }
        if (ALL && a.dgate) {
            float* to = a.parts > 1 ? a.partial + (4 * a.groups + blockIdx.x) * a.width : a.dgate + gate * a.width;
            put_sums<L>(dgate, cols, to, shared);
            dgate.clear();
        }
        begin = end > begin ? end : begin;
        if (begin >= last) break;
    }
    const auto at = [&](int sum) { return a.partial + (sum * a.groups + blockIdx.x) * a.width; };
    if (a.pre_w) {
        put_sums<L>(dpre_w, cols, at(0), shared);
        if (BIAS && a.pre_b) put_sums<L>(dpre_b, cols, at(1), shared);
    }
    if (ALL && a.post_w) {
        put_sums<L>(dpost_w, cols, at(2), shared);
        if (BIAS && a.post_b) put_sums<L>(dpost_b, cols, at(3), shared);
    }
}

// Adds partial rows: 32 columns a workgroup, 32 slices of the rows, always in the same
// order.  blockIdx.y: one of the four parameter gradients (rows = all groups), or 4 + gate
// (rows = that gate's parts).
struct NormOutputs { float* to[4]; };
constexpr int NORM_ADD_COLS = 32, NORM_ADD_SLICES = 32, NORM_ADD_BLOCK = NORM_ADD_COLS * NORM_ADD_SLICES;

__global__ __launch_bounds__(NORM_ADD_BLOCK) void norm_add_kernel(NormOutputs out, float* dgate, const float* partial,
                                                                  uint64_t groups, uint32_t parts, uint32_t width) {
    __shared__ float shared[NORM_ADD_SLICES][NORM_ADD_COLS];
    const uint32_t which = blockIdx.y, c = threadIdx.x % NORM_ADD_COLS, slice = threadIdx.x / NORM_ADD_COLS;
    const uint32_t col = blockIdx.x * NORM_ADD_COLS + c;
    float* to = which < 4 ? out.to[which] : dgate + (uint64_t)(which - 4) * width;
    if (!to) return;
    const float* from = partial + (which < 4 ? which * groups : 4 * groups + (uint64_t)(which - 4) * parts) * width + col;
    const uint32_t rows = which < 4 ? (uint32_t)groups : parts;
    float sum = 0.0f;
    if (col < width)
#pragma unroll 8
        for (uint32_t r = slice; r < rows; r += NORM_ADD_SLICES) sum += from[(uint64_t)r * width];
    shared[slice][c] = sum;
    __syncthreads();
    if (slice == 0 && col < width) {
        for (int i = 1; i < NORM_ADD_SLICES; ++i) sum += shared[i][c];
        to[col] = sum;
    }
}

// ------------------------------------------------------------------ host

// Checks what both directions share and fills the kernels' arguments; false if refused.
static bool norm_args(const okt_residual_norm* op, NormArgs& a) {
    if (!op || !known_dtype(op->dtype) || op->rows > NORM_MAX_ROWS || op->width < NORM_MIN_WIDTH || op->width > NORM_MAX_WIDTH) return false;
    if (op->kind != OKT_NORM_LAYER && op->kind != OKT_NORM_RMS) return false;
    if (!(op->eps >= 0.0f) || op->residual_scale != op->residual_scale) return false;
    if (!dropout_rule(op->dropout_p, a.drop)) return false;
    if (a.drop.bar != 65536u && (!op->d_seed || !aligned(op->d_seed, 8))) return false;
    if ((op->d_post_bias && !op->d_post_weight) || (op->d_pre_bias && !op->d_pre_weight)) return false;
    for (const float* p : {op->d_post_weight, op->d_post_bias, op->d_gate, op->d_pre_weight, op->d_pre_bias})
        if (!aligned(p, 16)) return false;
    const auto stride = [&](uint64_t s) { return s ? s : (uint64_t)op->width; };
    a.u_stride = stride(op->u_stride);
    a.x_stride = stride(op->x_stride);
    a.h_stride = stride(op->h_stride);
    a.y_stride = stride(op->y_stride);
    a.dh_stride = stride(op->dh_stride);
    a.dy_stride = stride(op->dy_stride);
    a.dx_stride = stride(op->dx_stride);
    a.du_stride = stride(op->du_stride);
    for (uint64_t s : {a.u_stride, a.x_stride, a.h_stride, a.y_stride, a.dh_stride, a.dy_stride, a.dx_stride, a.du_stride})
        if (s < op->width || s > (1ull << 20)) return false;
    a.rows = op->rows;
    a.width = op->width;
    a.site = op->site;
    a.eps = op->eps;
    a.alpha = op->residual_scale;
    a.inv_width = 1.0f / (float)op->width;
    a.layer = op->kind == OKT_NORM_LAYER;
    a.seed = op->d_seed;
    a.post_w = op->d_post_weight;
    a.post_b = op->d_post_bias;
    a.gate = op->d_gate;
    a.pre_w = op->d_pre_weight;
    a.pre_b = op->d_pre_bias;
    a.rows_per_gate = op->rows_per_gate == 0 || op->rows_per_gate > op->rows ? (op->rows ? op->rows : 1) : op->rows_per_gate;
    a.stats = nullptr;
    a.partial = a.dgate = nullptr;
    a.chunk = a.groups = 0;
    a.parts = 1;
    return true;
}

// Where two [rows, width] tensors share an element.  Rows of unlike strides that lie in the same stretch are taken to
// share one only where their first rows do.
static bool rows_overlap(const void* a, uint64_t a_stride, const void* b, uint64_t b_stride, uint64_t rows, uint64_t row_bytes, size_t e) {
    const uint64_t between = rows - 1;
    if (!a || !b || !overlap(a, between * a_stride * e + row_bytes, b, between * b_stride * e + row_bytes)) return false;
    if (rows == 1 || overlap(a, row_bytes, b, row_bytes)) return true;
    if (a_stride != b_stride) return false;
    const uint64_t step = a_stride * e, apart = (a < b ? (uintptr_t)b - (uintptr_t)a : (uintptr_t)a - (uintptr_t)b) % step;
    return apart < row_bytes || step - apart < row_bytes;
}

// An output may lie in an input's place, row by row, and nowhere else in it.
static bool misplaced(const void* out, uint64_t out_stride, const void* in, uint64_t in_stride, const NormArgs& a, size_t e) {
    if (out == in && (out_stride == in_stride || a.rows == 1)) return false;
    return rows_overlap(out, out_stride, in, in_stride, a.rows, a.width * e, e);
}

struct NormPointers { const void *u, *x, *h, *dh, *dy; void *out_h, *out_y, *dx, *du; };

template <typename T, typename L>
static void launch_norm(const NormArgs& a, const NormPointers& p, bool backward, unsigned groups, unsigned threads, hipStream_t s) {
    const dim3 grid(groups), block(threads);
    if (!backward) {
        hipLaunchKernelGGL((norm_forward_kernel<T, L>), grid, block, 0, s, a, (const T*)p.u, (const T*)p.x, (T*)p.out_h, (T*)p.out_y);
        return;
    }
    const bool bias = a.post_b || a.pre_b, drop = a.drop.bar != 65536u;
    auto* kernel = bias ? norm_backward_kernel<T, L, false, true, false> : norm_backward_kernel<T, L, false, false, false>;
    if constexpr (!(L::one && L::vecs == 2 && sizeof(T) == 4)) {           // norm_shape gives such a row another layout
        if (a.post_w || a.gate)
            kernel = drop ? (bias ? norm_backward_kernel<T, L, true, true, true> : norm_backward_kernel<T, L, true, false, true>)
                          : (bias ? norm_backward_kernel<T, L, true, true, false> : norm_backward_kernel<T, L, true, false, false>);
    }
    hipLaunchKernelGGL(kernel, grid, block, 0, s, a, (const T*)p.u, (const T*)p.h, (const T*)p.dh, (const T*)p.dy, (T*)p.dx, (T*)p.du);
}

template <typename T>
static void launch_norm_shape(const NormArgs& a, const NormPointers& p, bool backward, NormShape n, unsigned groups, hipStream_t s) {
    if (n.lanes == WAVE && n.vecs == 1) launch_norm<T, Layout<true, 1, 256>>(a, p, backward, groups, 256, s);
    else if (n.lanes == WAVE) launch_norm<T, Layout<true, 2, 256>>(a, p, backward, groups, 256, s);
    else if (n.vecs == 1) launch_norm<T, Layout<false, 1, 512>>(a, p, backward, groups, n.lanes, s);
    else launch_norm<T, Layout<false, 2, 512>>(a, p, backward, groups, n.lanes, s);
}

static void launch_norm_type(int dtype, const NormArgs& a, const NormPointers& p, bool backward, NormShape n, unsigned groups,
                             hipStream_t s) {
    if (dtype == OKT_F32) launch_norm_shape<float>(a, p, backward, n, groups, s);
    else if (dtype == OKT_BF16) launch_norm_shape<__bf16>(a, p, backward, n, groups, s);
    else launch_norm_shape<_Float16>(a, p, backward, n, groups, s);
}

}  // namespace okt

extern "C" {

size_t okt_residual_norm_workspace_bytes(uint64_t rows, uint32_t width, uint64_t rows_per_gate) {
    if (width < okt::NORM_MIN_WIDTH || width > okt::NORM_MAX_WIDTH || rows > okt::NORM_MAX_ROWS) return 0;
    const size_t need = okt::norm_ws_bytes(rows, width, rows_per_gate);
    return need ? need : 256;
}

int okt_residual_norm_forward(const okt_residual_norm* op, const void* d_u, const void* d_x, void* d_h_out, void* d_y_out,
                              float* d_stats_out, void* stream) {
    using namespace okt;
    NormArgs a;
    if (!norm_args(op, a)) return OKT_ERR_INVALID_ARG;
    if (a.rows == 0) return OKT_OK;
    if (!d_u || !d_x || (!d_h_out && !a.pre_w) || (a.pre_w && !d_y_out) || (!a.pre_w && d_y_out)) return OKT_ERR_INVALID_ARG;
    const size_t e = dtype_bytes(op->dtype);
    for (const void* p : {d_u, d_x, (const void*)d_h_out, (const void*)d_y_out})
        if (!aligned(p, e)) return OKT_ERR_INVALID_ARG;
    if (!aligned(d_stats_out, 16)) return OKT_ERR_INVALID_ARG;
    if (rows_overlap(d_h_out, a.h_stride, d_y_out, a.y_stride, a.rows, a.width * e, e) ||
        misplaced(d_h_out, a.h_stride, d_u, a.u_stride, a, e) || misplaced(d_h_out, a.h_stride, d_x, a.x_stride, a, e) ||
        misplaced(d_y_out, a.y_stride, d_u, a.u_stride, a, e) || misplaced(d_y_out, a.y_stride, d_x, a.x_stride, a, e)) return OKT_ERR_INVALID_ARG;
    a.stats = (float4*)d_stats_out;
    const NormShape shape = norm_shape(a.width, a.rows, op->dtype, false);
    const uint64_t at_once = rows_at_once(shape);
    const uint64_t want = (a.rows + at_once - 1) / at_once, most = (uint64_t)device_cus() * 8;
    timing_before((hipStream_t)stream);
    launch_norm_type(op->dtype, a, {d_u, d_x, nullptr, nullptr, nullptr, d_h_out, d_y_out, nullptr, nullptr}, false, shape,
                     (unsigned)(want < most ? want : most), (hipStream_t)stream);
    timing_after((hipStream_t)stream);
    return launch_status();
}

int okt_residual_norm_backward(const okt_residual_norm* op, const void* d_u, const void* d_h, const float* d_stats,
                               const void* d_dh, const void* d_dy, void* d_dx_out, void* d_du_out, float* d_dpost_weight_out,
                               float* d_dpost_bias_out, float* d_dgate_out, float* d_dpre_weight_out, float* d_dpre_bias_out,
                               void* d_ws, size_t ws_bytes, void* stream) {
    using namespace okt;
    NormArgs a;
    if (!norm_args(op, a)) return OKT_ERR_INVALID_ARG;
    if ((d_dpost_weight_out && !a.post_w) || (d_dpost_bias_out && !a.post_b) || (d_dgate_out && !a.gate) ||
        (d_dpre_weight_out && !a.pre_w) || (d_dpre_bias_out && !a.pre_b)) return OKT_ERR_INVALID_ARG;
    for (const float* p : {d_dpost_weight_out, d_dpost_bias_out, d_dgate_out, d_dpre_weight_out, d_dpre_bias_out})
        if (!aligned(p, 4)) return OKT_ERR_INVALID_ARG;
    const bool all = a.post_w || a.gate;
    if (a.rows) {
        if (!d_dx_out || !d_du_out || !d_stats || !aligned(d_stats, 16) || (all && !d_u)) return OKT_ERR_INVALID_ARG;
        if ((a.pre_w && (!d_h || !d_dy)) || (!a.pre_w && (d_dy || !d_dh))) return OKT_ERR_INVALID_ARG;
        const size_t e = dtype_bytes(op->dtype);
        for (const void* p : {d_u, d_h, d_dh, d_dy, (const void*)d_dx_out, (const void*)d_du_out})
            if (!aligned(p, e)) return OKT_ERR_INVALID_ARG;
        const struct { const void* p; uint64_t stride; } in[] = {{all ? d_u : nullptr, a.u_stride}, {a.pre_w ? d_h : nullptr, a.h_stride},
                                                                 {d_dh, a.dh_stride}, {d_dy, a.dy_stride}};
        for (const auto& t : in)
            if (misplaced(d_dx_out, a.dx_stride, t.p, t.stride, a, e) || misplaced(d_du_out, a.du_stride, t.p, t.stride, a, e)) return OKT_ERR_INVALID_ARG;
    }
    const NormShape shape = norm_shape(a.width, a.rows, op->dtype, all);
    const NormPlan plan = norm_plan(a.rows, a.rows_per_gate, rows_at_once(shape));
    if (!d_ws || !aligned(d_ws, 256) || ws_bytes < norm_ws_bytes(a.rows, a.width, a.rows_per_gate)) return OKT_ERR_WORKSPACE;
    if (a.rows && rows_overlap(d_dx_out, a.dx_stride, d_du_out, a.du_stride, a.rows, a.width * dtype_bytes(op->dtype), dtype_bytes(op->dtype)))
        return OKT_ERR_INVALID_ARG;
    a.stats = (float4*)d_stats;
    a.partial = (float*)d_ws;
    a.dgate = d_dgate_out;
    a.chunk = plan.chunk;
    a.groups = plan.groups;
    a.parts = plan.parts;
    const hipStream_t s = (hipStream_t)stream;
    if (a.rows) {
        timing_before(s);
        launch_norm_type(op->dtype, a, {d_u, nullptr, d_h, d_dh, d_dy, nullptr, nullptr, d_dx_out, d_du_out}, true,
                         shape, (unsigned)plan.groups, s);
        timing_after(s);
        if (const int status = launch_status()) return status;
    }
    NormOutputs out = {{d_dpre_weight_out, d_dpre_bias_out, d_dpost_weight_out, d_dpost_bias_out}};
    const bool gates = d_dgate_out && plan.parts != 1;
    if (out.to[0] || out.to[1] || out.to[2] || out.to[3] || gates)
        hipLaunchKernelGGL(norm_add_kernel, dim3((a.width + NORM_ADD_COLS - 1) / NORM_ADD_COLS, 4 + (gates ? (unsigned)plan.gates : 0)),
                           dim3(NORM_ADD_BLOCK), 0, s, out, d_dgate_out, (const float*)d_ws, plan.groups, plan.parts, a.width);
    return launch_status();
}

}  // extern "C"
