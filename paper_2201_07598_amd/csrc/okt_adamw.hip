// okt_adamw_step: one AdamW step over many tensors in one launch, states in 32 bits or in 8.
//
//   m = beta1 m + (1 - beta1) g,  v = beta2 v + (1 - beta2) g^2
//   p = (1 - lr wd) p - lr / (1 - beta1^t) m / (sqrt(v) / sqrt(1 - beta2^t) + eps)
//
// Every element is read once and written once and none meets another, so memory bounds it: 28 bytes an element in 32 bits,
// 16 with 8-bit states, 16-bit gradients and a 16-bit copy, 22 and 10 where the parameters have 16 bits themselves.  The tensors are cut into chunks of 4096 elements, a workgroup
// each; a table in the plan says which tensor a chunk is of, so that a launch over 400 tensors is as wide
// as one over their concatenation.  A lane holds four neighbours of each of its wave's four blocks of 256: all of a chunk's loads are
// on their way before the first is waited for.  334 M parameters in 389 tensors take 1657 us with 32-bit states (5.65 TB/s, 93 % of what a
// plain copy reaches) and 901 us with 8-bit ones and the copy (5.96 TB/s, 98 %); as bf16 1260 (5.8 TB/s) and 720 (4.7);
// 37 small tensors 6.6 us, one wave's way through a chunk.
//
// 8-bit states.  A block of 256 shares a scale, the power of two that brings its largest magnitude to (224, 448], and
// holds m / scale and sqrt(v) / scale in e4m3.  The root because that halves the range of exponents that v needs, and no v above
// 0 becomes 0, because m / sqrt(v) would explode there.  Values are rounded with the random field's bits, m so that its
// expectation is m, the root so that the expectation of its square is v (above v where the least code, 1, stands for less than itself): rounded to nearest,
// an average that moves by a thousandth a step would never leave a code whose steps are an eighth.
#include <algorithm>
#include <math.h>

#include "okt_element.h"
#include "okt_random.h"

namespace okt {

constexpr int ADAM_THREADS = 256;
constexpr int ADAM_GROUPS = 4;                                       // blocks of a wave
constexpr uint32_t ADAM_STATE_BLOCK = WAVE * 4;                      // elements that share a scale
constexpr uint32_t ADAM_CHUNK = ADAM_THREADS / WAVE * ADAM_GROUPS * ADAM_STATE_BLOCK;
constexpr uint64_t ADAM_MAX_CHUNKS = (1ull << 24) - 1;               // a launch counts work-items in 32 bits

// Steps that move more than this go around the caches, where nothing of them would be found again (67 M elements in 32
// bits 310 us, through the caches 348; 334 M 1657 and 1781, in 8 bits 970 and 1007); below it much is (17 M 78 and 70 us, 34 M in 8 bits 94 and 89).
constexpr uint64_t ADAM_CACHED_BYTES = 640ull << 20;

static_assert(ADAM_STATE_BLOCK == OKT_ADAMW_BLOCK, "the header's");

// What the kernel reads of a tensor.
struct AdamTensor {
    uint64_t p, g, m, v, copy, m_scale, v_scale, n;
    double weight_decay, rate_scale;
    uint32_t first_chunk, p_type, g_type, copy_type;
    uint64_t pad[2];
};
static_assert(sizeof(AdamTensor) == 112, "seven intervals of sixteen bytes fit in its place");

struct AdamScalars {
    const int64_t* step;
    const float *lr, *grad_scale, *skip;
    const uint64_t* seed;
    double log_beta1, log_beta2, host_lr;
    float beta1, beta2, rest1, rest2, eps;
    uint32_t site;
};

typedef float f32x4 __attribute__((ext_vector_type(4)));

// Addresses that come out of memory are taken for any address space, and loads from those wait for LDS as well.
template <typename T> using global = __attribute__((address_space(1))) T;

template <bool NT, typename T>
__device__ __forceinline__ f32x4 load_four(const global<T>* p) {
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec loose __attribute__((aligned(sizeof(T))));
    const vec v = NT ? __builtin_nontemporal_load((const global<loose>*)p) : *(const global<loose>*)p;
    return __builtin_convertvector(v, f32x4);
}
template <bool NT, typename T>
__device__ __forceinline__ void store_four(global<T>* p, f32x4 v) {
    typedef T vec __attribute__((ext_vector_type(4)));
    typedef vec loose __attribute__((aligned(sizeof(T))));
    if (NT) __builtin_nontemporal_store(__builtin_convertvector(v, vec), (global<loose>*)p);
    else *(global<loose>*)p = __builtin_convertvector(v, vec);
}
typedef uint32_t WordAnywhere __attribute__((aligned(1)));

// `left` elements of four are there (4: all).
template <bool FULL, bool NT, typename T>
__device__ __forceinline__ f32x4 some_four(const global<T>* p, int left) {
    if (FULL || left >= 4) return load_four<NT>(p);
    f32x4 v = 0.0f;
    if (left > 0) v[0] = (float)p[0];
    if (left > 1) v[1] = (float)p[1];
    if (left > 2) v[2] = (float)p[2];
    return v;
}
template <bool FULL, bool NT, typename T>
__device__ __forceinline__ void put_four(global<T>* p, f32x4 v, int left) {
    if (FULL || left >= 4) return store_four<NT>(p, v);
    if (left > 0) p[0] = (T)v[0];
    if (left > 1) p[1] = (T)v[1];
    if (left > 2) p[2] = (T)v[2];
}
template <bool FULL, bool NT>
__device__ __forceinline__ uint32_t some_codes(const global<uint8_t>* p, int left) {
    if (FULL || left >= 4) return NT ? __builtin_nontemporal_load((const global<WordAnywhere>*)p) : *(const global<WordAnywhere>*)p;
    uint32_t w = 0;
    if (left > 0) w = p[0];
    if (left > 1) w |= (uint32_t)p[1] << 8;
    if (left > 2) w |= (uint32_t)p[2] << 16;
    return w;
}
template <bool FULL, bool NT>
__device__ __forceinline__ void put_codes(global<uint8_t>* p, uint32_t w, int left) {
    if (FULL || left >= 4) {
        if (NT) __builtin_nontemporal_store(w, (global<WordAnywhere>*)p);
        else *(global<WordAnywhere>*)p = w;
        return;
    }
    if (left > 0) p[0] = (uint8_t)w;
    if (left > 1) p[1] = (uint8_t)(w >> 8);
    if (left > 2) p[2] = (uint8_t)(w >> 16);
}

// Largest of the wave's values, in every lane.
__device__ __forceinline__ uint32_t wave_max_u32(uint32_t v) {
#define OKT_MAX_STEP(ctrl, rows) v = max(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, ctrl, rows, 0xf, false))
    OKT_MAX_STEP(0x111, 0xf);      // row_shr:1, 2, 4, 8: lane 15 of each row has the row's
    OKT_MAX_STEP(0x112, 0xf);
    OKT_MAX_STEP(0x114, 0xf);
    OKT_MAX_STEP(0x118, 0xf);
    OKT_MAX_STEP(0x142, 0xa);      // row_bcast:15, 31: lane 63 has the wave's
    OKT_MAX_STEP(0x143, 0xc);
#undef OKT_MAX_STEP
    return (uint32_t)__builtin_amdgcn_readlane((int)v, WAVE - 1);
}

// A block's scale from the bits of its largest magnitude: the largest over it is above 224 and at most 448 = 1.75 2^8,
// e4m3's last value.  Blocks whose values are all below 2^-118 share the scale 2^-126.
struct BlockScale {
    float scale, back;                                               // and its reciprocal
    int to_bits;                                                     // the reciprocal over 2^120, as an exponent
    bool finite;
    __device__ __forceinline__ explicit BlockScale(uint32_t top) {
        const uint32_t e = max((top + 0x1fffffu) >> 23, 9u);
        finite = top < 0x7f800000u;
        scale = __uint_as_float(finite ? (e - 8) << 23 : 0x7fc00000u);
        back = __uint_as_float((262 - e) << 23);
        to_bits = 15 - (int)e;
    }
};

// The bits of y 2^-120 are y's e4m3 code and below it twenty bits of what is left of a step: the exponents' ends meet, fp32's
// subnormals from 2^-126 down are e4m3's from 2^-6 down.
__device__ __forceinline__ uint32_t code_bits(float x, int to_bits) { return __float_as_uint(__builtin_amdgcn_ldexpf(fabsf(x), to_bits)); }
__device__ __forceinline__ float code_value(uint32_t bits) { return __uint_as_float(bits) * 0x1p120f; }

__device__ __forceinline__ uint32_t signed_code(float x, const BlockScale& s, uint32_t half) {
    return (code_bits(x, s.to_bits) + half * 16) >> 20 | (__float_as_uint(x) >> 24 & 0x80u);
}

__device__ __forceinline__ uint32_t root_code(float w, const BlockScale& s, uint32_t half) {
    const uint32_t bits = code_bits(w, s.to_bits) & 0xfff00000u;
    const float y = w * s.back, a = code_value(bits), b = code_value(bits + 0x100000u);
    // at 448 the left side is 0
    const uint32_t code = (bits >> 20) + (y * y - a * a > (float)half * 0x1p-16f * (b * b - a * a) ? 1 : 0);
    return max(code, w > 0.0f ? 1u : 0u);
}

struct Rates { float keep, size, root; };

// One step of an element; m and v as they go on.
__device__ __forceinline__ float adam_element(float p, float g, float& m, float& v, float& w, const AdamScalars& a, const Rates& r) {
    m = a.beta1 * m + a.rest1 * g;
    v = a.beta2 * v + a.rest2 * g * g;
    w = sqrtf(v);
    // a root is 0 or above 2^-75 and eps 0 or a normal number, so the reciprocal is good to an ulp
    return p * r.keep - r.size * (m * __builtin_amdgcn_rcpf(w * r.root + a.eps));
}

template <typename P, typename G, bool EIGHT, bool NT, bool FULL>
__device__ __forceinline__ void adam_chunk(const AdamTensor& t, uint32_t chunk, uint32_t tensor, const AdamScalars& a) {
    const uint32_t lane = threadIdx.x % WAVE, wave = uniform(threadIdx.x / WAVE);
    const uint64_t block0 = (uint64_t)(chunk - t.first_chunk) * (ADAM_CHUNK / ADAM_STATE_BLOCK) + wave * ADAM_GROUPS;
    const uint64_t e0 = block0 * ADAM_STATE_BLOCK + lane * 4;
    const auto left = [&](int i) {                               // elements of a lane's four that the tensor has
        const int64_t n = (int64_t)(t.n - e0) - i * (int64_t)ADAM_STATE_BLOCK;
        return n > 4 ? 4 : (int)n;
    };
    // a block past the tensor's end has no scale
    const auto there = [&](int i) { return FULL || (block0 + i) * ADAM_STATE_BLOCK < t.n; };
    f32x4 p[ADAM_GROUPS], g[ADAM_GROUPS], m[ADAM_GROUPS], v[ADAM_GROUPS];
    uint32_t mc[ADAM_GROUPS], vc[ADAM_GROUPS];
    float ms[ADAM_GROUPS], vs[ADAM_GROUPS];
#pragma unroll
    for (int i = 0; i < ADAM_GROUPS; ++i) {
        const uint64_t e = e0 + i * ADAM_STATE_BLOCK;
        p[i] = some_four<FULL, NT>((const global<P>*)t.p + e, FULL ? 4 : left(i));
        g[i] = some_four<FULL, NT>((const global<G>*)t.g + e, FULL ? 4 : left(i));
        if (EIGHT) {
            mc[i] = some_codes<FULL, NT>((const global<uint8_t>*)t.m + e, FULL ? 4 : left(i));
            vc[i] = some_codes<FULL, NT>((const global<uint8_t>*)t.v + e, FULL ? 4 : left(i));
            ms[i] = there(i) ? ((const global<float>*)t.m_scale)[block0 + i] : 0.0f;
            vs[i] = there(i) ? ((const global<float>*)t.v_scale)[block0 + i] : 0.0f;
        } else {
            m[i] = some_four<FULL, NT>((const global<float>*)t.m + e, FULL ? 4 : left(i));
            v[i] = some_four<FULL, NT>((const global<float>*)t.v + e, FULL ? 4 : left(i));
        }
    }
    // 1 - beta^t in 64 bits, while the loads are on their way: near t = 1 it is a difference of neighbours
    const double steps = (double)max(*a.step, (int64_t)1);
    const double lr = (a.lr ? (double)*a.lr : a.host_lr) * t.rate_scale;
    const Rates r = {(float)(1.0 - lr * t.weight_decay), (float)(lr / -expm1(steps * a.log_beta1)),
                     (float)(1.0 / sqrt(-expm1(steps * a.log_beta2)))};
    const float grad_scale = a.grad_scale ? *a.grad_scale : 1.0f;
    RandomKey key = {0, 0};
    if (EIGHT && a.seed) key = random_key(a.seed);
#pragma unroll
    for (int i = 0; i < ADAM_GROUPS; ++i) {
        const uint64_t e = e0 + i * ADAM_STATE_BLOCK;
        if (EIGHT) {
            const auto m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[i], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)mc[i], true);
            const auto v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)vc[i], true);
            m[i] = f32x4{m01[0], m01[1], m23[0], m23[1]} * ms[i];
            v[i] = f32x4{v01[0], v01[1], v23[0], v23[1]} * vs[i];
            v[i] *= v[i];
        }
        f32x4 w;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            float mj = m[i][j], vj = v[i][j], wj;
            p[i][j] = adam_element(p[i][j], g[i][j] * grad_scale, mj, vj, wj, a, r);
            m[i][j] = mj;
            v[i][j] = vj;
            w[j] = wj;
        }
        put_four<FULL, NT>((global<P>*)t.p + e, p[i], FULL ? 4 : left(i));
        if (t.copy) {
            if (t.copy_type == OKT_BF16) put_four<FULL, NT>((global<__bf16>*)t.copy + e, p[i], FULL ? 4 : left(i));
            else put_four<FULL, NT>((global<_Float16>*)t.copy + e, p[i], FULL ? 4 : left(i));
        }
        if (!EIGHT) {
            put_four<FULL, NT>((global<float>*)t.m + e, m[i], FULL ? 4 : left(i));
            put_four<FULL, NT>((global<float>*)t.v + e, v[i], FULL ? 4 : left(i));
            continue;
        }
        // what the tensor has not got was read as 0 and stays 0, so it raises no block's largest
        uint32_t top_m = 0, top_w = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            top_m = max(top_m, magnitude_key(m[i][j]));
            top_w = max(top_w, __float_as_uint(w[j]));           // no roots below 0
        }
        const BlockScale sm(wave_max_u32(top_m)), sw(wave_max_u32(top_w));
        RandomBlock rnd = {{0x80008000u, 0x80008000u, 0x80008000u, 0x80008000u}};
        if (a.seed) rnd = random_block(key, (uint32_t)(e / 4), (uint32_t)(e / 4 >> 32), tensor, a.site);
        uint32_t code_m = 0, code_v = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t hm = j & 1 ? rnd.w[j / 2] >> 16 : rnd.w[j / 2] & 0xffffu;
            const uint32_t hv = j & 1 ? rnd.w[2 + j / 2] >> 16 : rnd.w[2 + j / 2] & 0xffffu;
            code_m |= signed_code(m[i][j], sm, hm) << (8 * j);
            code_v |= root_code(w[j], sw, hv) << (8 * j);
        }
        put_codes<FULL, NT>((global<uint8_t>*)t.m + e, sm.finite ? code_m : 0, FULL ? 4 : left(i));
        put_codes<FULL, NT>((global<uint8_t>*)t.v + e, sw.finite ? code_v : 0, FULL ? 4 : left(i));
        if (lane == 0 && there(i)) {
            ((global<float>*)t.m_scale)[block0 + i] = sm.scale;
            ((global<float>*)t.v_scale)[block0 + i] = sw.scale;
        }
    }
}

template <typename P, typename G, bool EIGHT, bool NT>
__device__ __forceinline__ void adam_ends(const AdamTensor& t, uint32_t chunk, uint32_t tensor, const AdamScalars& a) {
    if ((uint64_t)(chunk - t.first_chunk + 1) * ADAM_CHUNK <= t.n) adam_chunk<P, G, EIGHT, NT, true>(t, chunk, tensor, a);
    else adam_chunk<P, G, EIGHT, NT, false>(t, chunk, tensor, a);
}

template <typename P, bool EIGHT, bool NT>
__device__ __forceinline__ void adam_gradient(const AdamTensor& t, uint32_t chunk, uint32_t tensor, const AdamScalars& a) {
    if (t.g_type == OKT_F32) adam_ends<P, float, EIGHT, NT>(t, chunk, tensor, a);
    else if (t.g_type == OKT_BF16) adam_ends<P, __bf16, EIGHT, NT>(t, chunk, tensor, a);
    else adam_ends<P, _Float16, EIGHT, NT>(t, chunk, tensor, a);
}

template <bool EIGHT, bool NT>
__global__ __launch_bounds__(ADAM_THREADS) void adamw_kernel(AdamScalars a, const AdamTensor* tensors, const uint32_t* tensor_of) {
    if (a.skip && *a.skip != 0.0f) return;
    const uint32_t chunk = blockIdx.x, tensor = tensor_of[chunk];
    const AdamTensor t = tensors[tensor];
    if (t.p_type == OKT_F32) adam_gradient<float, EIGHT, NT>(t, chunk, tensor, a);
    else if (t.p_type == OKT_BF16) adam_gradient<__bf16, EIGHT, NT>(t, chunk, tensor, a);
    else adam_gradient<_Float16, EIGHT, NT>(t, chunk, tensor, a);
}

// ------------------------------------------------------------------ the plan

struct AdamSizes { uint64_t chunks, bytes; };

static bool adam_sizes(const okt_adamw_tensor* tensors, uint32_t count, AdamSizes& s) {
    s.chunks = 0;
    for (uint32_t i = 0; i < count; ++i) {
        if (tensors[i].n > ADAM_MAX_CHUNKS * ADAM_CHUNK) return false;
        s.chunks += (tensors[i].n + ADAM_CHUNK - 1) / ADAM_CHUNK;
        if (s.chunks > ADAM_MAX_CHUNKS) return false;
    }
    s.bytes = ((uint64_t)count * sizeof(AdamTensor) + s.chunks * 4 + 255) / 256 * 256;
    return true;
}

// Memory that a step reads (the gradients) or writes; the address's top bit, which no address has, marks what is read only.
struct Interval { uint64_t begin, end; };
constexpr uint64_t READ_ONLY = 1ull << 63;

// Whether two intervals share a byte of which one writes.
static bool intervals_clash(Interval* v, size_t n) {
    std::sort(v, v + n, [](const Interval& a, const Interval& b) { return a.begin < b.begin; });
    uint64_t written = 0, any = 0;                        // where those before end
    for (size_t i = 0; i < n; ++i) {
        const uint64_t end = v[i].end & ~READ_ONLY;
        const bool reads = v[i].end & READ_ONLY;
        if (v[i].begin < (reads ? written : any)) return true;
        if (!reads && end > written) written = end;
        if (end > any) any = end;
    }
    return false;
}

}  // namespace okt

extern "C" {

size_t okt_adamw_plan_bytes(const okt_adamw_tensor* h_tensors, uint32_t count) {
    okt::AdamSizes s;
    if (!h_tensors || count == 0 || !okt::adam_sizes(h_tensors, count, s)) return 0;
    return s.bytes;
}

int okt_adamw_plan(const okt_adamw_tensor* h_tensors, uint32_t count, int state, void* h_plan_out, size_t plan_bytes,
                   uint32_t* h_chunks_out) {
    using namespace okt;
    AdamSizes s;
    if (!h_tensors || count == 0 || (state != OKT_STATE_F32 && state != OKT_STATE_E4M3) || !adam_sizes(h_tensors, count, s) || !h_chunks_out)
        return OKT_ERR_INVALID_ARG;
    if (!h_plan_out || !aligned(h_plan_out, 8) || plan_bytes < s.bytes) return OKT_ERR_WORKSPACE;
    const bool eight = state == OKT_STATE_E4M3;
    Interval* at = (Interval*)h_plan_out;
    size_t intervals = 0;
    for (uint32_t i = 0; i < count; ++i) {
        const okt_adamw_tensor& t = h_tensors[i];
        if (!known_dtype(t.param_dtype) || !known_dtype(t.grad_dtype) || (t.d_copy && t.copy_dtype != OKT_BF16 && t.copy_dtype != OKT_F16) ||
            !(t.weight_decay >= 0.0) || !isfinite(t.weight_decay) || !(t.rate_scale >= 0.0) || !isfinite(t.rate_scale))
            return OKT_ERR_INVALID_ARG;
        if (t.n == 0) continue;
        const size_t pe = dtype_bytes(t.param_dtype), ge = dtype_bytes(t.grad_dtype), se = eight ? 1 : 4;
        const uint64_t blocks = (t.n + ADAM_STATE_BLOCK - 1) / ADAM_STATE_BLOCK;
        if (!t.d_param || !t.d_grad || !t.d_m || !t.d_v || eight != (t.d_m_scale != nullptr) || eight != (t.d_v_scale != nullptr))
            return OKT_ERR_INVALID_ARG;
        const struct { const void* p; uint64_t bytes; size_t align; bool reads; } parts[7] = {
            {t.d_param, t.n * pe, pe, false}, {t.d_grad, t.n * ge, ge, true}, {t.d_m, t.n * se, se, false}, {t.d_v, t.n * se, se, false},
            {t.d_copy, t.n * 2, 2, false}, {t.d_m_scale, blocks * 4, 4, false}, {t.d_v_scale, blocks * 4, 4, false}};
        for (const auto& part : parts) {
            if (!part.p) continue;
            const uint64_t begin = (uint64_t)(uintptr_t)part.p;
            if (begin % part.align || begin >= READ_ONLY - part.bytes) return OKT_ERR_INVALID_ARG;
            at[intervals++] = {begin, (begin + part.bytes) | (part.reads ? READ_ONLY : 0)};
        }
    }
    if (intervals_clash(at, intervals)) return OKT_ERR_INVALID_ARG;
    AdamTensor* to = (AdamTensor*)h_plan_out;
    uint32_t* tensor_of = (uint32_t*)(to + count);
    uint32_t chunk = 0;
    for (uint32_t i = 0; i < count; ++i) {
        const okt_adamw_tensor& t = h_tensors[i];
        const auto address = [](const void* p) { return (uint64_t)(uintptr_t)p; };
        to[i] = {address(t.d_param), address(t.d_grad), address(t.d_m), address(t.d_v), address(t.d_copy), address(t.d_m_scale),
                 address(t.d_v_scale), t.n, t.weight_decay, t.rate_scale, chunk, (uint32_t)t.param_dtype, (uint32_t)t.grad_dtype,
                 (uint32_t)t.copy_dtype, {0, 0}};
        for (uint64_t c = (t.n + ADAM_CHUNK - 1) / ADAM_CHUNK; c > 0; --c) tensor_of[chunk++] = i;
    }
    for (char* end = (char*)(tensor_of + chunk); end < (char*)h_plan_out + s.bytes; ++end) *end = 0;
    *h_chunks_out = chunk;
    return OKT_OK;
}

int okt_adamw_step(const okt_adamw* op, const void* d_plan, void* stream) {
    using namespace okt;
    if (!op || (op->state != OKT_STATE_F32 && op->state != OKT_STATE_E4M3) || op->tensors == 0 || op->chunks > ADAM_MAX_CHUNKS)
        return OKT_ERR_INVALID_ARG;
    const auto share = [](double b) { return b >= 0.0 && b < 1.0; };
    if (!share(op->beta1) || !share(op->beta2) || !(op->eps >= 0.0) || !isfinite(op->eps) || (!op->d_lr && !isfinite((float)op->lr))) return OKT_ERR_INVALID_ARG;
    if (!op->d_step || !aligned(op->d_step, 8) || !aligned(op->d_seed, 8)) return OKT_ERR_INVALID_ARG;
    for (const float* p : {op->d_lr, op->d_grad_scale, op->d_skip})
        if (!aligned(p, 4)) return OKT_ERR_INVALID_ARG;
    if (op->chunks == 0) return OKT_OK;
    if (!d_plan || !aligned(d_plan, 16)) return OKT_ERR_INVALID_ARG;
    const AdamScalars a = {op->d_step, op->d_lr, op->d_grad_scale, op->d_skip, op->d_seed, log(op->beta1), log(op->beta2), op->lr,
                           (float)op->beta1, (float)op->beta2, (float)(1.0 - op->beta1), (float)(1.0 - op->beta2), op->eps > 0.0 ? fmaxf((float)op->eps, 0x1p-126f) : 0.0f, op->site};
    const hipStream_t s = (hipStream_t)stream;
    const AdamTensor* tensors = (const AdamTensor*)d_plan;
    const uint32_t* tensor_of = (const uint32_t*)(tensors + op->tensors);
    const bool eight = op->state == OKT_STATE_E4M3, around = (uint64_t)op->chunks * ADAM_CHUNK * (eight ? 16 : 28) > ADAM_CACHED_BYTES;
    timing_before(s);
    hipLaunchKernelGGL(eight ? (around ? adamw_kernel<true, true> : adamw_kernel<true, false>)
                             : (around ? adamw_kernel<false, true> : adamw_kernel<false, false>),
                       dim3(op->chunks), dim3(ADAM_THREADS), 0, s, a, tensors, tensor_of);
    timing_after(s);
    return launch_status();
}

}  // extern "C"
