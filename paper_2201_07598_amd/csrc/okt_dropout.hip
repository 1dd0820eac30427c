// okt_dropout: y = x * 65536 / bar where the random field keeps the place, else 0.
//
// The mask is never stored: 2n elements of traffic and nothing else.  A thread owns
// DROP_GROUPS groups of eight neighbours, and a group is one block of the random field, so
// that one evaluation of the generator (14 wide multiplications) serves eight elements
// and 16 bytes are read and written at once.  Bound by memory: 67.1 M bf16 elements take 47 us from call
// to call, 5.7 TB/s of 268 MB (the kernel 39), a vector of one workgroup 5.7 us, 1.4 of them in the kernel.
#include "okt_element.h"
#include "okt_random.h"

namespace okt {

constexpr int DROP_BLOCK = 256;
constexpr int DROP_GROUPS = 4;
constexpr uint64_t DROP_TILE = (uint64_t)DROP_BLOCK * DROP_GROUPS * 8;      // elements per workgroup
constexpr uint64_t DROP_MAX_N = ((1ull << 24) - 1) * DROP_TILE;              // a launch counts work-items in 32 bits

template <typename T>
__device__ __forceinline__ f32x8 drop_eight(f32x8 v, uint64_t group, RandomKey key, uint32_t site, DropoutRule rule) {
    const RandomBlock b = random_block(key, (uint32_t)group, (uint32_t)(group >> 32), 0, site);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = kept(b, i, rule.bar) ? v[i] * rule.scale : 0.0f;
    return v;
}

template <typename T>
__global__ __launch_bounds__(DROP_BLOCK) void dropout_kernel(const T* x, T* y, uint64_t n, const uint64_t* d_seed,
                                                             uint32_t site, DropoutRule rule) {
    const RandomKey key = random_key(d_seed);
    const uint64_t group0 = (uint64_t)blockIdx.x * (DROP_BLOCK * DROP_GROUPS) + threadIdx.x;
    if (((uint64_t)blockIdx.x + 1) * DROP_TILE <= n) {
        f32x8 v[DROP_GROUPS];
#pragma unroll
        for (int g = 0; g < DROP_GROUPS; ++g) v[g] = load_eight(x + (group0 + g * DROP_BLOCK) * 8);
#pragma unroll
        for (int g = 0; g < DROP_GROUPS; ++g) {
            const uint64_t group = group0 + g * DROP_BLOCK;
            store_eight(y + group * 8, drop_eight<T>(v[g], group, key, site, rule));
        }
        return;
    }
    for (int g = 0; g < DROP_GROUPS; ++g) {                     // the last workgroup
        const uint64_t group = group0 + g * DROP_BLOCK;
        if (group * 8 + 8 <= n) {
            store_eight(y + group * 8, drop_eight<T>(load_eight(x + group * 8), group, key, site, rule));
        } else if (group * 8 < n) {
            const int count = (int)(n - group * 8);
            f32x8 v = 0.0f;
            if (n >= 8) v = __builtin_convertvector(skip_elements<T>(raw_eight(x + n - 8), 8 - count), f32x8);
            else for (int i = 0; i < count; ++i) v[i] = (float)x[i];
            store_some(y + group * 8, drop_eight<T>(v, group, key, site, rule), count);
        }
    }
}

template <typename T>
static int launch_dropout(const void* x, void* y, uint64_t n, const uint64_t* d_seed, uint32_t site, DropoutRule rule,
                          hipStream_t stream) {
    timing_before(stream);
    hipLaunchKernelGGL(dropout_kernel<T>, dim3((unsigned)((n + DROP_TILE - 1) / DROP_TILE)), dim3(DROP_BLOCK), 0, stream,
                       (const T*)x, (T*)y, n, d_seed, site, rule);
    timing_after(stream);
    return launch_status();
}

}  // namespace okt

extern "C" int okt_dropout(const void* d_x, void* d_y, uint64_t n, int dtype, double p, const uint64_t* d_seed,
                           uint32_t site, void* stream) {
    using namespace okt;
    DropoutRule rule;
    if (!known_dtype(dtype) || !dropout_rule(p, rule) || n > DROP_MAX_N) return OKT_ERR_INVALID_ARG;
    if (n == 0) return OKT_OK;
    if (!d_x || !d_y || !d_seed || !aligned(d_x, 16) || !aligned(d_y, 16) || !aligned(d_seed, 8)) return OKT_ERR_INVALID_ARG;
    if (d_x != d_y && overlap(d_x, n * dtype_bytes(dtype), d_y, n * dtype_bytes(dtype))) return OKT_ERR_INVALID_ARG;
    const hipStream_t s = (hipStream_t)stream;
    if (dtype == OKT_F32) return launch_dropout<float>(d_x, d_y, n, d_seed, site, rule, s);
    if (dtype == OKT_BF16) return launch_dropout<__bf16>(d_x, d_y, n, d_seed, site, rule, s);
    return launch_dropout<_Float16>(d_x, d_y, n, d_seed, site, rule, s);
}
