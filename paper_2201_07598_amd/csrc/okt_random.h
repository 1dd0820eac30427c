// The counter-based random field that dropout, the residual norm and attention draw
// from: Philox4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as
// 1, 2, 3", SC'11) with seven rounds, the least its authors found to pass every test they ran.  The
// key is the caller's 64-bit seed, the counter (c0, c1, c2, site) names a block of eight
// 16-bit values; nothing of it is stored, the backward pass draws the same values again.
#ifndef OKT_RANDOM_H
#define OKT_RANDOM_H

#include "okt_device.h"

namespace okt {

constexpr int RANDOM_ROUNDS = 7;

struct RandomBlock { uint32_t w[4]; };     // value 2i + h is half h (0 = low) of word i

// The caller's seed, which is the same for every lane.
struct RandomKey { uint32_t lo, hi; };

__device__ __forceinline__ RandomKey random_key(const uint64_t* d_seed) {
    const uint64_t s = *d_seed;
    return {uniform((uint32_t)s), uniform((uint32_t)(s >> 32))};
}

// a ^ b ^ c in one instruction.
__device__ __forceinline__ uint32_t xor_three(uint32_t a, uint32_t b, uint32_t c) {
    return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96);
}

__device__ __forceinline__ RandomBlock random_block(RandomKey key, uint32_t c0, uint32_t c1, uint32_t c2,
                                                    uint32_t site) {
    uint32_t c3 = site;
#pragma unroll
    for (int r = 0; r < RANDOM_ROUNDS; ++r) {
        const uint64_t a = (uint64_t)c0 * 0xD2511F53u, b = (uint64_t)c2 * 0xCD9E8D57u;
        c0 = xor_three((uint32_t)(b >> 32), c1, key.lo);
        c1 = (uint32_t)b;
        c2 = xor_three((uint32_t)(a >> 32), c3, key.hi);
        c3 = (uint32_t)a;
        key.lo += 0x9E3779B9u;
        key.hi += 0xBB67AE85u;
    }
    return {{c0, c1, c2, c3}};
}

// What a probability p of dropping comes to: values below `bar` are kept (bar 65536 keeps
// all, 0 none), and what is kept is multiplied by 65536 / bar, the reciprocal of the share
// that is really kept, so that the expectation is that of the input whatever p rounds to.
struct DropoutRule { uint32_t bar; float scale; };

inline bool dropout_rule(double p, DropoutRule& rule) {
    if (!(p >= 0.0 && p <= 1.0)) return false;             // a NaN is refused, too
    rule.bar = (uint32_t)((1.0 - p) * 65536.0 + 0.5);
    rule.scale = rule.bar ? (float)(65536.0 / rule.bar) : 0.0f;
    return true;
}

// Whether value i (0..7, known when compiled) of a block is kept.
__device__ __forceinline__ bool kept(const RandomBlock& b, int i, uint32_t bar) {
    const uint32_t w = b.w[i >> 1];
    return ((i & 1) ? w >> 16 : w & 0xffffu) < bar;
}

}  // namespace okt

#endif
