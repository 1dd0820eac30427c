// okt_norm_rotary_forward / _backward: a norm of each head of queries and keys and the rotation of its pairs by position.
//
//   n = (x - m) r w  (or x),   y_a = n_a cos - n_b sin,   y_b = n_a sin + n_b cos   for the pair (a, b) of angle position * freq
//
// Backward the rotation is turned back, then dx = r (d w - h mean(h d w) - mean(d w)), h = (x - m) r, and dw = sum d h.
// Every element comes once and goes once (backward: two come, one goes), so memory bounds it: 8 x 4096 tokens of 16 + 4 heads of 128 bf16
// with both norms take 67 us forward and 101 backward, 5.0 TB/s, 83 % of what a plain copy reaches; a token by itself 9 us, which is the host.
//
// A workgroup takes a few tokens.  First its threads make the cosines and sines of those tokens, each once, in LDS, where
// all heads find them: the angle in fp64 turns of which the whole ones are dropped, because a position of 10^5 times a frequency
// has lost 2^-7 of a turn in fp32.  Then lanes take heads: eight elements a lane as two fours, which are the two halves of four pairs (or
// four adjacent pairs), so a pair never leaves its lane and a norm's sums cross 8, 16 or 32 lanes inside the vector unit.
#include <algorithm>
#include <initializer_list>
#include <math.h>

#include "okt_attention_layout.h"
#include "okt_element.h"

namespace okt {

constexpr int ROT_THREADS = 256;
constexpr uint32_t ROT_MAX_DIM = 256, ROT_MAX_TOKENS = 32;           // of a workgroup at a time
constexpr uint32_t ROT_ANGLES = 1024;                                // a workgroup's tokens times pairs
constexpr uint32_t ROT_BACKWARD_GROUPS = 1024;
// Heads of a lane that are on their way together.  (8 x 4096 tokens of 16 + 4 heads of 128 bf16, backward: one 119 us, two 108, four 128,
// which takes registers of half the waves; forward two and four 74, one 83.  fp32, of twice the registers: backward one 191, two 202, forward one 129 and
// two 125; 3 x 1001 tokens of 12 + 12 heads of 80 22.0 and 28.4, forward 12.5 and 12.7.)
template <typename T> constexpr int ROT_AHEAD = 2;
template <> constexpr int ROT_AHEAD<float> = 1;
// Calls that move more than this go around the caches, of which they would find nothing again (the sizes above: 73 and 108 us through them, 68 and 102
// around); what smaller ones write, attention finds there.
constexpr uint64_t ROT_CACHED_BYTES = 256ull << 20;

struct HeadStrides { uint64_t batch, row; uint32_t head; };          // in elements

struct RotTensor {                                                   // queries or keys
    uint32_t heads;
    uint32_t step_tokens, step_heads;                                // what a lane's next head is further than its last one
    const float* weight;
    HeadStrides in, d, out;
};

struct RotArgs {
    uint32_t tokens, tiles;
    uint32_t dim, rot, tile, groups, pair_shift;                     // tokens a tile; workgroups (backward); pairs rounded up, as a shift
    Divider length;
    int kind;
    uint32_t axes;
    bool adjacent;
    float eps, share;                                                // share: 1 / dim
    const float* inv_freq;
    const int32_t* positions;
    uint64_t position_stride[2];
    RotTensor t[2];
    float* partial;
    uint8_t axis_of_pair[ROT_MAX_DIM / 2];
};

struct RotPointers { const void* x[2]; const void* d[2]; void* out[2]; };

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Four neighbours as they lie in memory, at the alignment of an element.
template <typename T> using Four = T __attribute__((ext_vector_type(4)));
template <typename T> using LooseFour = T __attribute__((ext_vector_type(4), aligned(sizeof(T))));
template <bool NT, typename T> __device__ __forceinline__ Four<T> raw_four(const T* p) {
    return NT ? __builtin_nontemporal_load(reinterpret_cast<const LooseFour<T>*>(p)) : *reinterpret_cast<const LooseFour<T>*>(p);
}
template <typename T> __device__ __forceinline__ f32x4 wide_four(Four<T> v) { return __builtin_convertvector(v, f32x4); }
template <bool NT, typename T> __device__ __forceinline__ void store_four(T* p, f32x4 v) {
    if (NT) __builtin_nontemporal_store(__builtin_convertvector(v, Four<T>), reinterpret_cast<LooseFour<T>*>(p));
    else *reinterpret_cast<LooseFour<T>*>(p) = __builtin_convertvector(v, Four<T>);
}

__device__ __forceinline__ f32x4 fma_four(f32x4 a, f32x4 b, f32x4 c) {
    return f32x4{fmaf(a[0], b[0], c[0]), fmaf(a[1], b[1], c[1]), fmaf(a[2], b[2], c[2]), fmaf(a[3], b[3], c[3])};
}

// 1 / sqrt, to an ulp: the unit's instruction takes no subnormal numbers.
__device__ __forceinline__ float reciprocal_root(float v) {
    const bool tiny = v < 0x1p-96f;
    return __builtin_amdgcn_rsqf(tiny ? v * 0x1p64f : v) * (tiny ? 0x1p32f : 1.0f);
}

// Sum over LANES (8, 16 or 32) neighbouring lanes, in each of them.
template <int LANES>
__device__ __forceinline__ float head_sum(float v) {
#define OKT_SUM_STEP(ctrl) v += __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v), ctrl, 0xf, 0xf, true))
    OKT_SUM_STEP(0xB1);           // quad_perm [1, 0, 3, 2]
    OKT_SUM_STEP(0x4E);           // quad_perm [2, 3, 0, 1]
    OKT_SUM_STEP(0x141);          // row_half_mirror: the other four of eight
    if (LANES >= 16) OKT_SUM_STEP(0x140);     // row_mirror: the other eight of sixteen
#undef OKT_SUM_STEP
    if (LANES >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
        v = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return v;
}

struct Eights { f32x4 a, b; };                                       // four pairs: first and second of each

__device__ __forceinline__ float sum_of(const Eights& x) {
    const f32x4 s = x.a + x.b;
    return (s[0] + s[1]) + (s[2] + s[3]);
}
__device__ __forceinline__ float dot_of(const Eights& x, const Eights& y) {
    const f32x4 s = fma_four(x.a, y.a, x.b * y.b);
    return (s[0] + s[1]) + (s[2] + s[3]);
}

struct TokenPlace { uint64_t in[2], d[2], out[2]; };

// What a workgroup's threads share about its tokens.
struct RotShared {
    f32x4 cosine[ROT_ANGLES / 4], sine[ROT_ANGLES / 4];              // [token][pair], dim / 2 pairs; the unrotated are turned by 0
    TokenPlace place[ROT_MAX_TOKENS];
};

// Where the tokens of a tile lie.
template <bool BACKWARD>
__device__ __forceinline__ void rot_places(const RotArgs& a, RotShared& s, uint32_t first, uint32_t count) {
    if (threadIdx.x >= count) return;
    const uint32_t token = first + threadIdx.x, b = quotient(token, a.length), i = token - b * a.length.by;
    TokenPlace p;
#pragma unroll
    for (int n = 0; n < 2; ++n) {
        p.in[n] = b * a.t[n].in.batch + i * a.t[n].in.row;
        if (BACKWARD) p.d[n] = b * a.t[n].d.batch + i * a.t[n].d.row;
        p.out[n] = b * a.t[n].out.batch + i * a.t[n].out.row;
    }
    s.place[threadIdx.x] = p;
}

// Cosines and sines of their pairs, each once.
__device__ __forceinline__ void rot_angles(const RotArgs& a, RotShared& s, uint32_t first, uint32_t count) {
    const uint32_t pairs = a.dim / 2, j = threadIdx.x & ((1u << a.pair_shift) - 1);
    if (j >= pairs) return;
    const bool turns = j < a.rot / 2;
    const double freq = turns ? (double)a.inv_freq[j] * 0.15915494309189533577 : 0.0;        // in turns: 1 / 2 pi
    const uint32_t axis = turns ? a.axis_of_pair[j] : 0;
    for (uint32_t t = threadIdx.x >> a.pair_shift; t < count; t += ROT_THREADS >> a.pair_shift) {
        float c = 1.0f, d = 0.0f;
        if (turns) {
            const uint32_t token = first + t, b = quotient(token, a.length), i = token - b * a.length.by;
            const int32_t position = a.positions ? a.positions[b * a.position_stride[0] + i * a.position_stride[1] + axis] : (int32_t)i;
            const double angle = (double)position * freq;
            sincospif((float)(2.0 * (angle - rint(angle))), &d, &c);
        }
        reinterpret_cast<float*>(s.cosine)[t * pairs + j] = c;
        reinterpret_cast<float*>(s.sine)[t * pairs + j] = d;
    }
}

// Where a lane's two fours lie in a head, and back and forth between them and pairs.
struct LanePlace {
    uint32_t first, second, unit;
    bool there, turned;                                              // unrotated elements pass: their partners' infinities times a sine of 0 are NaN
    template <int LANES>
    static __device__ __forceinline__ LanePlace of(const RotArgs& a) {
        const uint32_t unit = threadIdx.x % LANES;
        const bool apart = !a.adjacent && unit < a.rot / 8;
        return {apart ? unit * 4 : unit * 8, apart ? a.rot / 2 + unit * 4 : unit * 8 + 4, unit, unit * 8 < a.dim, unit * 8 < a.rot};
    }
    template <bool NT, typename T>
    __device__ __forceinline__ void store(T* head, const Eights& v, bool adjacent) const {
        f32x4 x = v.a, y = v.b;
        if (adjacent) {
            x = f32x4{v.a[0], v.b[0], v.a[1], v.b[1]};
            y = f32x4{v.a[2], v.b[2], v.a[3], v.b[3]};
        }
        store_four<NT>(head + first, x);
        store_four<NT>(head + second, y);
    }
    static __device__ __forceinline__ Eights pairs(Eights v, bool adjacent) {
        if (!adjacent) return v;
        return {f32x4{v.a[0], v.a[2], v.b[0], v.b[2]}, f32x4{v.a[1], v.a[3], v.b[1], v.b[3]}};
    }
    __device__ __forceinline__ Eights weight(const float* w, bool adjacent) const {
        if (!w || !there) return {1.0f, 1.0f};
        return pairs({wide_four<float>(raw_four<false>(w + first)), wide_four<float>(raw_four<false>(w + second))}, adjacent);
    }
};

// Heads of a tile in the order in which a group of lanes takes them.
struct HeadWalk {
    uint32_t token, head;
    __device__ __forceinline__ void next(const RotTensor& t) {
        token += t.step_tokens;
        head += t.step_heads;
        if (head >= t.heads) {
            head -= t.heads;
            ++token;
        }
    }
    template <int LANES>
    static __device__ __forceinline__ HeadWalk begin(const RotTensor& t) {
        HeadWalk w = {0, threadIdx.x / LANES};
        while (w.head >= t.heads) {
            w.head -= t.heads;
            ++w.token;
        }
        return w;
    }
};

// A lane's parts of the next heads of its group, as they lie in memory.
template <typename T, int N, bool BACKWARD, bool NT>
struct HeadBatch {
    static constexpr int AHEAD = ROT_AHEAD<T>;
    HeadWalk at[AHEAD];
    Four<T> x[AHEAD][2], d[BACKWARD ? AHEAD : 1][2];
    __device__ __forceinline__ void load(const RotArgs& a, const RotShared& s, const LanePlace& lane, HeadWalk& walk, uint32_t count, const T* px, const T* pd) {
        const RotTensor& t = a.t[N];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            at[k] = walk;
            x[k][0] = x[k][1] = Four<T>{};
            if (BACKWARD) d[k][0] = d[k][1] = Four<T>{};
            if (walk.token < count && lane.there) {
                if (!BACKWARD || t.weight) {
                    const T* head = px + s.place[walk.token].in[N] + (uint64_t)walk.head * t.in.head;
                    x[k][0] = raw_four<NT>(head + lane.first);
                    x[k][1] = raw_four<NT>(head + lane.second);
                }
                if (BACKWARD) {
                    const T* head = pd + s.place[walk.token].d[N] + (uint64_t)walk.head * t.d.head;
                    d[k][0] = raw_four<NT>(head + lane.first);
                    d[k][1] = raw_four<NT>(head + lane.second);
                }
            }
            walk.next(t);
        }
    }
};

// x less its mean (layer norm) and the reciprocal of its deviation.
template <int LANES>
__device__ __forceinline__ float head_statistics(const RotArgs& a, const LanePlace& at, Eights& v) {
    if (a.kind == OKT_NORM_LAYER) {
        const float mean = head_sum<LANES>(sum_of(v)) * a.share;
        if (at.there) {
            v.a -= mean;
            v.b -= mean;
        }
    }
    return reciprocal_root(fmaf(head_sum<LANES>(dot_of(v, v)), a.share, a.eps));
}

template <typename T, int LANES, int N, bool NT>
struct Forward {
    typedef HeadBatch<T, N, false, NT> Batch;
    LanePlace at;
    HeadWalk walk;
    Batch now;
    const T* x;
    __device__ __forceinline__ Forward(const RotArgs& a, const RotShared& s, uint32_t count, const T* from) : at(LanePlace::of<LANES>(a)), x(from) {
        if (a.t[N].heads == 0) return;
        walk = HeadWalk::begin<LANES>(a.t[N]);
        now.load(a, s, at, walk, count, x, nullptr);
    }
    __device__ __forceinline__ void run(const RotArgs& a, const RotShared& s, uint32_t count, T* out) {
        const RotTensor& t = a.t[N];
        if (t.heads == 0) return;
        const Eights w = at.weight(t.weight, a.adjacent);
        while (now.at[0].token < count) {
#pragma unroll
            for (int k = 0; k < Batch::AHEAD; ++k) {
                if (now.at[k].token >= count) break;            // the same for all lanes of a head
                Eights v = LanePlace::pairs({wide_four<T>(now.x[k][0]), wide_four<T>(now.x[k][1])}, a.adjacent);
                const uint32_t angle = now.at[k].token * (a.dim / 8) + (at.there ? at.unit : 0);
                f32x4 c = s.cosine[angle], d = s.sine[angle];
                if (t.weight) {
                    const float r = head_statistics<LANES>(a, at, v);
                    v.a *= w.a;
                    v.b *= w.b;
                    c *= r;
                    d *= r;
                }
                Eights y = {fma_four(v.a, c, -(v.b * d)), fma_four(v.a, d, v.b * c)};
                if (a.rot < a.dim && !at.turned) y = {v.a * c, v.b * c};
                if (at.there) at.template store<NT>(out + s.place[now.at[k].token].out[N] + (uint64_t)now.at[k].head * t.out.head, y, a.adjacent);
            }
            now.load(a, s, at, walk, count, x, nullptr);
        }
    }
};

template <typename T, int LANES, bool NT>
__global__ __launch_bounds__(ROT_THREADS) void norm_rotary_forward_kernel(RotArgs a, RotPointers p) {
    __shared__ RotShared s;
    const uint32_t first = blockIdx.x * a.tile, count = min(a.tokens - first, a.tile);
    rot_places<false>(a, s, first, count);
    __syncthreads();
    Forward<T, LANES, 0, NT> q(a, s, count, (const T*)p.x[0]);           // on their way while the angles are made
    rot_angles(a, s, first, count);
    __syncthreads();
    q.run(a, s, count, (T*)p.out[0]);
    Forward<T, LANES, 1, NT> k(a, s, count, (const T*)p.x[1]);
    k.run(a, s, count, (T*)p.out[1]);
}

template <typename T, int LANES, int N, bool NT>
struct Backward {
    typedef HeadBatch<T, N, true, NT> Batch;
    LanePlace at;
    HeadWalk walk;
    Batch now;
    const T *x, *dy;
    __device__ __forceinline__ Backward(const RotArgs& a, const RotShared& s, uint32_t count, const T* px, const T* pd)
        : at(LanePlace::of<LANES>(a)), x(px), dy(pd) {
        if (a.t[N].heads == 0) return;
        walk = HeadWalk::begin<LANES>(a.t[N]);
        now.load(a, s, at, walk, count, x, dy);
    }
    __device__ __forceinline__ void run(const RotArgs& a, const RotShared& s, uint32_t count, T* out, Eights& dw) {
        const RotTensor& t = a.t[N];
        if (t.heads == 0) return;
        const Eights w = at.weight(t.weight, a.adjacent);
        while (now.at[0].token < count) {
#pragma unroll
            for (int k = 0; k < Batch::AHEAD; ++k) {
                if (now.at[k].token >= count) break;
                const uint32_t angle = now.at[k].token * (a.dim / 8) + (at.there ? at.unit : 0);
                const f32x4 c = s.cosine[angle], e = s.sine[angle];
                const Eights d = LanePlace::pairs({wide_four<T>(now.d[k][0]), wide_four<T>(now.d[k][1])}, a.adjacent);
                Eights g = {fma_four(d.a, c, d.b * e), fma_four(d.b, c, -(d.a * e))};
                if (a.rot < a.dim && !at.turned) g = d;
                if (t.weight) {
                    Eights v = LanePlace::pairs({wide_four<T>(now.x[k][0]), wide_four<T>(now.x[k][1])}, a.adjacent);
                    const float r = head_statistics<LANES>(a, at, v);
                    v.a *= r;                                   // h
                    v.b *= r;
                    dw.a = fma_four(g.a, v.a, dw.a);
                    dw.b = fma_four(g.b, v.b, dw.b);
                    g.a *= w.a;
                    g.b *= w.b;
                    const float along = head_sum<LANES>(dot_of(g, v)) * a.share;
                    if (a.kind == OKT_NORM_LAYER) {
                        const float level = head_sum<LANES>(sum_of(g)) * a.share;
                        g.a -= level;
                        g.b -= level;
                    }
                    g.a = r * fma_four(v.a, f32x4(-along), g.a);
                    g.b = r * fma_four(v.b, f32x4(-along), g.b);
                }
                if (at.there) at.template store<NT>(out + s.place[now.at[k].token].out[N] + (uint64_t)now.at[k].head * t.out.head, g, a.adjacent);
            }
            now.load(a, s, at, walk, count, x, dy);
        }
    }
};

// A workgroup's sums of a weight's gradient, over its lanes of one unit; in the order of the elements of a head.
template <int LANES>
__device__ __forceinline__ void rot_sums(const RotArgs& a, float* sums, const Eights& dw, float* to) {
    const LanePlace at = LanePlace::of<LANES>(a);
    float v[8] = {dw.a[0], dw.a[1], dw.a[2], dw.a[3], dw.b[0], dw.b[1], dw.b[2], dw.b[3]};
#pragma unroll
    for (int i = 0; i < 8; ++i)
#pragma unroll
        for (int m = LANES; m < WAVE; m <<= 1) v[i] += __shfl_xor(v[i], m, WAVE);
    if (threadIdx.x % WAVE < LANES && at.there)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            // element i of the pairs' order in the head's
            const uint32_t e = a.adjacent ? at.unit * 8 + 2 * (i % 4) + i / 4 : (i < 4 ? at.first + i : at.second + i - 4);
            sums[threadIdx.x / WAVE * ROT_MAX_DIM + e] = v[i];
        }
    __syncthreads();
    for (uint32_t e = threadIdx.x; e < a.dim; e += ROT_THREADS) {
        float sum = 0.0f;
#pragma unroll
        for (int wave = 0; wave < ROT_THREADS / WAVE; ++wave) sum += sums[wave * ROT_MAX_DIM + e];
        to[e] = sum;
    }
}

template <typename T, int LANES, bool NT>
__global__ __launch_bounds__(ROT_THREADS) void norm_rotary_backward_kernel(RotArgs a, RotPointers p) {
    __shared__ RotShared s;
    __shared__ float sums[2][ROT_MAX_DIM * (ROT_THREADS / WAVE)];
    Eights dw[2] = {{0.0f, 0.0f}, {0.0f, 0.0f}};
    for (uint32_t tile = blockIdx.x; tile < a.tiles; tile += a.groups) {
        const uint32_t first = tile * a.tile, count = min(a.tokens - first, a.tile);
        rot_places<true>(a, s, first, count);
        __syncthreads();
        Backward<T, LANES, 0, NT> q(a, s, count, (const T*)p.x[0], (const T*)p.d[0]);
        rot_angles(a, s, first, count);
        __syncthreads();
        q.run(a, s, count, (T*)p.out[0], dw[0]);
        Backward<T, LANES, 1, NT> k(a, s, count, (const T*)p.x[1], (const T*)p.d[1]);
        k.run(a, s, count, (T*)p.out[1], dw[1]);
        __syncthreads();
    }
    if (!a.partial) return;
#pragma unroll
    for (int n = 0; n < 2; ++n)
        rot_sums<LANES>(a, sums[n], dw[n], a.partial + ((uint64_t)n * a.groups + blockIdx.x) * a.dim);
}

// Adds the workgroups' sums, always in the same order: sixteen columns by 64 parts a workgroup.
constexpr int ROT_ADD_COLS = 16, ROT_ADD_THREADS = 1024;
struct RotGradients { float* to[2]; };
__global__ __launch_bounds__(ROT_ADD_THREADS) void norm_rotary_add_kernel(const float* partial, uint32_t groups, uint32_t dim, RotGradients g) {
    constexpr int PARTS = ROT_ADD_THREADS / ROT_ADD_COLS;
    __shared__ float sums[PARTS][ROT_ADD_COLS];
    const uint32_t n = blockIdx.y, part = threadIdx.x / ROT_ADD_COLS, col = threadIdx.x % ROT_ADD_COLS, e = blockIdx.x * ROT_ADD_COLS + col;
    float sum = 0.0f;
    if (e < dim)
#pragma unroll 8
        for (uint32_t k = part; k < groups; k += PARTS) sum += partial[((uint64_t)n * groups + k) * dim + e];
    sums[part][col] = sum;
    __syncthreads();
    if (part != 0 || e >= dim || !g.to[n]) return;
#pragma unroll
    for (int k = 1; k < PARTS; ++k) sum += sums[k][col];
    g.to[n][e] = sum;
}

// ------------------------------------------------------------------ host

static uint32_t rot_lanes(uint32_t dim) { return dim <= 64 ? 8 : dim <= 128 ? 16 : 32; }

// Tokens a workgroup takes at a time: eight heads a lane, but no fewer workgroups than fill the chip four times, and
// what the shared memory holds.
static uint32_t rot_tile(uint64_t tokens, uint32_t heads, uint32_t dim) {
    const uint64_t at_once = ROT_THREADS / rot_lanes(dim), wanted = (8 * at_once + heads - 1) / heads;
    const uint64_t spread = (tokens + 1023) / 1024, room = ROT_ANGLES / (dim / 2);
    uint64_t t = wanted;
    for (const uint64_t most : {spread, room, (uint64_t)ROT_MAX_TOKENS}) t = most < t ? most : t;
    return t ? (uint32_t)t : 1;
}
static uint32_t rot_groups(uint64_t tiles) { return (uint32_t)(tiles < ROT_BACKWARD_GROUPS ? tiles : ROT_BACKWARD_GROUPS); }

static bool rot_sizes(uint32_t batch, uint32_t length, uint32_t heads, uint32_t kv_heads, uint32_t dim) {
    return heads <= 1u << 16 && kv_heads <= 1u << 16 && heads + kv_heads > 0 && dim >= 8 && dim <= ROT_MAX_DIM && dim % 8 == 0 &&
           (uint64_t)batch * length < 1ull << 24;
}

static bool rot_args(const okt_norm_rotary* op, RotArgs& a) {
    if (!op || !rot_sizes(op->batch, op->length, op->heads, op->kv_heads, op->head_dim) || !known_dtype(op->dtype)) return false;
    if (op->rot_dim > op->head_dim || op->rot_dim % 8 != 0 || op->axes < 1 || op->axes > 8) return false;
    if (op->kind != OKT_NORM_LAYER && op->kind != OKT_NORM_RMS) return false;
    if (!(op->eps >= 0.0f) || !isfinite(op->eps)) return false;
    if (op->rot_dim && (!op->d_inv_freq || !aligned(op->d_inv_freq, 4))) return false;
    if (!aligned(op->d_positions, 4) || (!op->d_positions && op->axes != 1)) return false;
    for (const float* w : {op->d_q_weight, op->d_k_weight})
        if (!aligned(w, 4)) return false;
    for (uint32_t j = 0; j < op->rot_dim / 2; ++j) {
        if (op->axis_of_pair[j] >= op->axes) return false;
        a.axis_of_pair[j] = op->axis_of_pair[j];
    }
    a.tokens = op->batch * op->length;
    a.length = divider(a.tokens ? op->length : 1);                   // a length without a batch may be any
    a.dim = op->head_dim;
    a.share = 1.0f / (float)op->head_dim;
    a.pair_shift = 2;
    while (1u << a.pair_shift < op->head_dim / 2) ++a.pair_shift;
    a.rot = op->rot_dim;
    a.kind = op->kind;
    a.axes = op->axes;
    a.adjacent = op->adjacent != 0;
    a.eps = op->eps;
    a.inv_freq = op->d_inv_freq;
    a.positions = op->d_positions;
    a.position_stride[0] = op->position_stride[0];
    a.position_stride[1] = op->position_stride[1];
    for (const uint64_t* s : {op->q_stride, op->k_stride, op->q_out_stride, op->k_out_stride, op->dq_stride, op->dk_stride})
        if (s[0] > 1ull << 40 || s[1] > 1ull << 40 || s[2] > 1ull << 30) return false;
    const auto strides = [](const uint64_t* s) { return HeadStrides{s[0], s[1], (uint32_t)s[2]}; };
    const uint32_t step = ROT_THREADS / rot_lanes(op->head_dim);
    const auto steps = [&](uint32_t heads, bool rest) { return heads == 0 ? 0 : rest ? step % heads : step / heads; };
    a.t[0] = {op->heads, steps(op->heads, false), steps(op->heads, true), op->d_q_weight,
              strides(op->q_stride), strides(op->dq_stride), strides(op->q_out_stride)};
    a.t[1] = {op->kv_heads, steps(op->kv_heads, false), steps(op->kv_heads, true), op->d_k_weight,
              strides(op->k_stride), strides(op->dk_stride), strides(op->k_out_stride)};
    a.partial = nullptr;
    if (a.tokens == 0) return true;
    a.tile = rot_tile(a.tokens, op->heads + op->kv_heads, op->head_dim);
    a.tiles = (a.tokens + a.tile - 1) / a.tile;
    a.groups = rot_groups(a.tiles);
    return true;
}

struct Placed { const void* p; HeadStrides s; uint32_t heads; };

// Steps along an axis of a tensor, or of the place of one of its heads less that of another's.
struct Axis { int64_t stride, least, most; };
constexpr uint64_t ROT_FARTHEST = 1ull << 50;                        // elements: no memory has so many
constexpr int ROT_TRIES = 1 << 14;

// Elements from a tensor's first to behind its last one, where `n` are together and every axis makes so many steps of a stride; ROT_FARTHEST
// where that is more.
struct Steps { uint64_t count, stride; };
static uint64_t extent(uint64_t n, std::initializer_list<Steps> axes) {
    for (const Steps& t : axes)
        if (t.count && t.stride) n = t.stride < (ROT_FARTHEST - n) / t.count ? n + t.count * t.stride : ROT_FARTHEST;
    return n;
}
static uint64_t extent(const RotArgs& a, const HeadStrides& s, uint32_t heads) {
    const uint32_t length = a.length.by, batch = a.tokens / length;
    return extent(a.dim, {{batch - 1, s.batch}, {length - 1, s.row}, {heads - 1, s.head}});
}

// Whether `apart` elements are some steps along the axes, each axis' within its size, and less than a head's length besides. The axes by falling
// stride: of each, the numbers of steps come into question whose rest those behind it can reach, which are two or fewer where a stride is more
// than they reach together. Where strides lie otherwise there may be many; after `tries` of them all the answer is yes.
static bool reachable(int64_t apart, const Axis* axes, int n, int64_t dim, int& tries) {
    if (n == 0) return apart > -dim && apart < dim;
    const int64_t stride = axes->stride;
    if (stride == 0) return reachable(apart, axes + 1, n - 1, dim, tries);
    int64_t low = apart - (dim - 1), high = apart + dim - 1;         // of what this axis' steps have to make
    for (int i = 1; i < n; ++i) {
        low -= axes[i].most * axes[i].stride;
        high -= axes[i].least * axes[i].stride;
    }
    if (high < axes->least * stride || low > axes->most * stride) return false;
    const int64_t first = low <= axes->least * stride ? axes->least : low / stride + (low % stride > 0);
    const int64_t last = high >= axes->most * stride ? axes->most : high / stride - (high % stride < 0);
    for (int64_t k = first; k <= last; ++k) {
        if (n == 1 || tries-- <= 0) return true;                     // the steps of the last axis were chosen so
        if (reachable(apart - k * stride, axes + 1, n - 1, dim, tries)) return true;
    }
    return false;
}

static void by_stride(Axis (&axes)[3]) {
    std::sort(axes, axes + 3, [](const Axis& p, const Axis& q) { return p.stride > q.stride; });
}

// An output of which two heads share an element: some steps along the axes, the first of them forward, lead less than a head's length away.
static bool shares_places(const RotArgs& a, const HeadStrides& s, uint32_t heads) {
    const int64_t batch = a.tokens / a.length.by, length = a.length.by;
    if ((batch > 1 && s.batch < a.dim) || (length > 1 && s.row < a.dim) || (heads > 1 && s.head < a.dim)) return true;
    if (extent(a, s, heads) >= ROT_FARTHEST) return true;
    const auto axis = [](uint64_t stride, int64_t size) { return Axis{(int64_t)(size > 1 ? stride : 0), 1 - size, size - 1}; };
    Axis axes[3] = {axis(s.batch, batch), axis(s.row, length), axis(s.head, heads)};
    by_stride(axes);
    int tries = ROT_TRIES;
    for (int n = 0; n < 3 && axes[n].stride; ++n) {
        Axis forward[3];
        std::copy(axes, axes + 3, forward);
        forward[n].least = 1;
        if (reachable(0, forward + n, 3 - n, a.dim, tries)) return true;
    }
    return false;
}

static uint64_t placed_bytes(const RotArgs& a, const Placed& t, size_t e) { return extent(a, t.s, t.heads) * e; }

// What a call reads beside the heads: weights, frequencies, positions.  Outputs are held apart from those by first and last element.
static bool over_parameters(const RotArgs& a, const void* out, uint64_t bytes) {
    const struct { const void* p; uint64_t bytes; } t[] = {
        {a.t[0].weight, 4ull * a.dim}, {a.t[1].weight, 4ull * a.dim}, {a.rot ? a.inv_freq : nullptr, 2ull * a.rot},
        {a.tokens && a.rot ? a.positions : nullptr,
         a.tokens ? 4 * extent(a.axes, {{a.tokens / a.length.by - 1, a.position_stride[0]}, {a.length.by - 1, a.position_stride[1]}}) : 0}};
    for (const auto& x : t)
        if (x.p && overlap(out, bytes, x.p, x.bytes)) return true;
    return false;
}

// Whether an output and another tensor share an element, one in the very place of the other aside, which the caller sees.  Where
// their strides are alike, as parts of one projection's are, by their heads; else by their first and last elements.
static bool clash(const RotArgs& a, const Placed& x, const Placed& y, size_t e) {
    if (!x.p || !y.p || !x.heads || !y.heads) return false;
    const uint64_t batch = a.tokens / a.length.by, length = a.length.by;
    if (!overlap(x.p, placed_bytes(a, x, e), y.p, placed_bytes(a, y, e))) return false;
    if (extent(a, x.s, x.heads) >= ROT_FARTHEST || extent(a, y.s, y.heads) >= ROT_FARTHEST) return true;
    if ((batch > 1 && x.s.batch != y.s.batch) || (length > 1 && x.s.row != y.s.row) || (x.heads > 1 && y.heads > 1 && x.s.head != y.s.head)) return true;
    const int64_t bytes = (int64_t)((uintptr_t)y.p - (uintptr_t)x.p);
    const int64_t b = (int64_t)batch - 1, l = (int64_t)length - 1;
    Axis axes[3] = {{(int64_t)(batch > 1 ? x.s.batch : 0), -b, b}, {(int64_t)(length > 1 ? x.s.row : 0), -l, l},
                    {(int64_t)(x.heads > 1 ? x.s.head : y.heads > 1 ? y.s.head : 0), 1 - (int64_t)y.heads, (int64_t)x.heads - 1}};
    by_stride(axes);
    int tries = ROT_TRIES;
    return reachable(bytes / (int64_t)e, axes, 3, a.dim, tries);
}
static bool same(const RotArgs& a, const Placed& x, const Placed& y) {
    return x.p == y.p && (x.s.batch == y.s.batch || a.tokens == a.length.by) && (x.s.row == y.s.row || a.length.by == 1) &&
           (x.s.head == y.s.head || x.heads == 1) && x.heads == y.heads;
}

template <typename T, int LANES>
static void launch_rot(const RotArgs& a, const RotPointers& p, bool backward, hipStream_t s) {
    const bool around = (uint64_t)a.tokens * (a.t[0].heads + a.t[1].heads) * a.dim * sizeof(T) * (backward ? 3 : 2) > ROT_CACHED_BYTES;
    if (backward)
        hipLaunchKernelGGL((around ? norm_rotary_backward_kernel<T, LANES, true> : norm_rotary_backward_kernel<T, LANES, false>), dim3(a.groups),
                           dim3(ROT_THREADS), 0, s, a, p);
    else
        hipLaunchKernelGGL((around ? norm_rotary_forward_kernel<T, LANES, true> : norm_rotary_forward_kernel<T, LANES, false>), dim3(a.tiles),
                           dim3(ROT_THREADS), 0, s, a, p);
}
template <typename T>
static void launch_rot_lanes(const RotArgs& a, const RotPointers& p, bool backward, hipStream_t s) {
    const uint32_t lanes = rot_lanes(a.dim);
    if (lanes == 8) launch_rot<T, 8>(a, p, backward, s);
    else if (lanes == 16) launch_rot<T, 16>(a, p, backward, s);
    else launch_rot<T, 32>(a, p, backward, s);
}
static int launch_rot_type(int dtype, const RotArgs& a, const RotPointers& p, bool backward, hipStream_t s) {
    timing_before(s);
    if (dtype == OKT_F32) launch_rot_lanes<float>(a, p, backward, s);
    else if (dtype == OKT_BF16) launch_rot_lanes<__bf16>(a, p, backward, s);
    else launch_rot_lanes<_Float16>(a, p, backward, s);
    timing_after(s);
    return launch_status();
}

}  // namespace okt

extern "C" {

size_t okt_norm_rotary_workspace_bytes(uint32_t batch, uint32_t length, uint32_t heads, uint32_t kv_heads, uint32_t head_dim) {
    using namespace okt;
    if (!rot_sizes(batch, length, heads, kv_heads, head_dim)) return 0;
    const uint64_t tokens = (uint64_t)batch * length;
    if (tokens == 0) return 256;
    const uint32_t tile = rot_tile(tokens, heads + kv_heads, head_dim);
    return ((size_t)rot_groups((tokens + tile - 1) / tile) * 2 * head_dim * 4 + 255) / 256 * 256;
}

int okt_norm_rotary_forward(const okt_norm_rotary* op, const void* d_q, const void* d_k, void* d_q_out, void* d_k_out, void* stream) {
    using namespace okt;
    RotArgs a;
    if (!rot_args(op, a)) return OKT_ERR_INVALID_ARG;
    if (a.tokens == 0) return OKT_OK;
    const size_t e = dtype_bytes(op->dtype);
    const RotPointers p = {{d_q, d_k}, {nullptr, nullptr}, {d_q_out, d_k_out}};
    Placed in[2], out[2];
    for (int n = 0; n < 2; ++n) {
        in[n] = {p.x[n], a.t[n].in, a.t[n].heads};
        out[n] = {p.out[n], a.t[n].out, a.t[n].heads};
        if (!a.t[n].heads) continue;
        if (!p.x[n] || !p.out[n] || !aligned(p.x[n], e) || !aligned(p.out[n], e) || shares_places(a, a.t[n].out, a.t[n].heads)) return OKT_ERR_INVALID_ARG;
        if (over_parameters(a, p.out[n], placed_bytes(a, out[n], e))) return OKT_ERR_INVALID_ARG;
    }
    if (clash(a, out[0], out[1], e)) return OKT_ERR_INVALID_ARG;
    for (int n = 0; n < 2; ++n)
        for (int m = 0; m < 2; ++m)
            if (!(n == m && same(a, out[n], in[m])) && clash(a, out[n], in[m], e)) return OKT_ERR_INVALID_ARG;
    return launch_rot_type(op->dtype, a, p, false, (hipStream_t)stream);
}

int okt_norm_rotary_backward(const okt_norm_rotary* op, const void* d_q, const void* d_k, const void* d_dq, const void* d_dk,
                             void* d_dq_out, void* d_dk_out, float* d_dq_weight_out, float* d_dk_weight_out, void* d_ws,
                             size_t ws_bytes, void* stream) {
    using namespace okt;
    RotArgs a;
    if (!rot_args(op, a)) return OKT_ERR_INVALID_ARG;
    RotGradients g = {{d_dq_weight_out, d_dk_weight_out}};
    const size_t e = dtype_bytes(op->dtype);
    const RotPointers p = {{d_q, d_k}, {d_dq, d_dk}, {d_dq_out, d_dk_out}};
    Placed in[2], d[2], out[2];
    for (int n = 0; n < 2; ++n) {
        if (!aligned(g.to[n], 4) || (g.to[n] && (!a.t[n].weight || !a.t[n].heads))) return OKT_ERR_INVALID_ARG;
        in[n] = {a.t[n].weight ? p.x[n] : nullptr, a.t[n].in, a.t[n].heads};
        d[n] = {p.d[n], a.t[n].d, a.t[n].heads};
        out[n] = {p.out[n], a.t[n].out, a.t[n].heads};
        if (!a.t[n].heads || a.tokens == 0) continue;
        if ((a.t[n].weight && !p.x[n]) || !p.d[n] || !p.out[n] || !aligned(p.x[n], e) || !aligned(p.d[n], e) || !aligned(p.out[n], e) ||
            shares_places(a, a.t[n].out, a.t[n].heads)) return OKT_ERR_INVALID_ARG;
        if (over_parameters(a, p.out[n], placed_bytes(a, out[n], e))) return OKT_ERR_INVALID_ARG;
    }
    for (float* to : g.to) {                                         // of the weights, written by the second launch
        if (!to) continue;
        if (over_parameters(a, to, 4ull * a.dim)) return OKT_ERR_INVALID_ARG;
        for (int n = 0; n < 2 && a.tokens; ++n)
            for (const Placed& t : {in[n], d[n], out[n]})
                if (t.p && t.heads && overlap(to, 4ull * a.dim, t.p, placed_bytes(a, t, e))) return OKT_ERR_INVALID_ARG;
    }
    if (g.to[0] && g.to[1] && overlap(g.to[0], 4ull * a.dim, g.to[1], 4ull * a.dim)) return OKT_ERR_INVALID_ARG;
    const bool sums = g.to[0] || g.to[1];
    if (a.tokens) {
        if (clash(a, out[0], out[1], e)) return OKT_ERR_INVALID_ARG;
        for (int n = 0; n < 2; ++n)
            for (int m = 0; m < 2; ++m)
                if ((!(n == m && same(a, out[n], in[m])) && clash(a, out[n], in[m], e)) ||
                    (!(n == m && same(a, out[n], d[m])) && clash(a, out[n], d[m], e))) return OKT_ERR_INVALID_ARG;
        if (sums && (!d_ws || !aligned(d_ws, 256) || ws_bytes < (size_t)a.groups * 2 * a.dim * 4)) return OKT_ERR_WORKSPACE;
        if (sums) a.partial = (float*)d_ws;
        if (const int status = launch_rot_type(op->dtype, a, p, true, (hipStream_t)stream)) return status;
    }
    if (sums)
        hipLaunchKernelGGL(norm_rotary_add_kernel, dim3((a.dim + ROT_ADD_COLS - 1) / ROT_ADD_COLS, 2), dim3(ROT_ADD_THREADS), 0, (hipStream_t)stream,
                           (const float*)d_ws, a.tokens ? a.groups : 0, a.dim, g);
    return sums ? launch_status() : OKT_OK;
}

}  // extern "C"
