// Tiles of matrix products on the matrix units: C[m][n] = sum over k of A(m, k) B(n, k) with 16-bit operands and fp32 sums.
//
// A workgroup has a tile of C, each of its waves MT x NT squares of 32 x 32 of it, as the unit's 32 x 32 x 16 steps leave them:
// lane l holds column n = l % 32 and, because rows of A are handed over in the order that makes it so, its sixteen
// elements are the neighbours m = 16 (l / 32) + r.  What goes out row by row of n is then contiguous in a lane.
//
// Operands pass through LDS in pieces of 64 k, fetched straight from memory into one of two buffers while the other one is multiplied, and
// lie in memory either way: with k contiguous (KMajor), or with k from row to row (Transposed), which the transposing LDS reads turn.  A
// fetch of a wave is 1024 bytes, eight rows of 128: whole cache lines.  Inside such a block the sixteen-byte chunks of a row are
// exchanged by an xor that makes the sixteen lanes of a read, in whichever order they read the rows, hit all banks once.
#ifndef OKT_PRODUCT_H
#define OKT_PRODUCT_H

#include "okt_attention.h"
#include "okt_product_layout.h"

namespace okt {

constexpr int PRODUCT_K = 64;                       // of a piece

// An operand's rows from `first` on, `rows` of them in the tensor, `bytes` from row to row.
struct OperandSource {
    uint64_t at, left;                              // address of the next piece, bytes from there to the tensor's end
    __device__ __forceinline__ i32x4 buffer() const {
        return {(int)uniform((uint32_t)at), (int)uniform((uint32_t)(at >> 32)), (int)uniform(left < OUTSIDE ? (uint32_t)left : OUTSIDE), 0x00020000};
    }
    __device__ __forceinline__ void advance(uint64_t by) {
        at += by;
        left = left > by ? left - by : 0;
    }
};

// ROWS rows (m or n) of 64 k each.  ORDERED: as A.
template <typename T, int ROWS, int WAVES, bool ORDERED>
struct KMajor {
    static constexpr int LOADS = ROWS / 8 / WAVES, BYTES = ROWS * PRODUCT_K * 2;
    static_assert(LOADS % 4 == 0, "a wave's blocks begin at a multiple of four");
    OperandSource from;
    uint32_t at[LOADS], read[4];

    // `end`: of the tensor's last row
    __device__ __forceinline__ KMajor(const T* tile, const T* end, uint32_t row_bytes) {
        const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
        from = {(uint64_t)tile, (uint64_t)end - (uint64_t)tile};
#pragma unroll
        for (int i = 0; i < LOADS; ++i) at[i] = ((wave * LOADS + i) * 8 + lane / 8) * row_bytes + kmajor_chunk<ORDERED>(lane, i) * 16;
#pragma unroll
        for (uint32_t s = 0; s < 4; ++s) read[s] = kmajor_read<ORDERED>(lane, s);
    }
    // `there`: k of this piece that the tensor has
    __device__ __forceinline__ void fetch(uint32_t lds, uint32_t there) {
        const uint32_t to = lds + uniform(threadIdx.x / WAVE) * (LOADS * 1024);
        const i32x4 buffer = from.buffer();
        if (there >= PRODUCT_K) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) fetch_to_lds(to + i * 1024, at[i], buffer);
        } else {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) fetch_to_lds(to + i * 1024, kmajor_chunk<ORDERED>(threadIdx.x % WAVE, i) * 8 < there ? at[i] : OUTSIDE, buffer);
        }
        from.advance(PRODUCT_K * 2);
    }
    __device__ __forceinline__ frag<T> operand(const char* piece, int square, int s) const {
        return *reinterpret_cast<const frag<T>*>(piece + read[s] + square * KMAJOR_SQUARE);
    }
};

// COLS columns (m or n) of 64 rows k each.
template <typename T, int COLS, int WAVES, bool ORDERED>
struct Transposed {
    static constexpr int LOADS = COLS / 8 / WAVES, BYTES = COLS * PRODUCT_K * 2;
    OperandSource from;
    uint64_t step;
    uint32_t at[LOADS], read[2];

    // `columns`: how many the tensor has from the tile's first on
    __device__ __forceinline__ Transposed(const T* tile, const T* end, uint64_t row_bytes, uint32_t columns) {
        const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
        from = {(uint64_t)tile, (uint64_t)end > (uint64_t)tile ? (uint64_t)end - (uint64_t)tile : 0};
        step = PRODUCT_K * row_bytes;
        const uint32_t r = lane / 8, c = transposed_chunk(lane);
#pragma unroll
        for (int i = 0; i < LOADS; ++i) {
            const uint32_t block = wave * LOADS + i, col = block / 8 * 64 + c * 8;
            at[i] = col < columns ? (block % 8 * 8 + r) * (uint32_t)row_bytes + col * 2 : OUTSIDE;
        }
#pragma unroll
        for (uint32_t half = 0; half < 2; ++half) read[half] = transposed_read<ORDERED>(lane, half);
    }
    __device__ __forceinline__ void fetch(uint32_t lds, uint32_t) {
        const uint32_t to = lds + uniform(threadIdx.x / WAVE) * (LOADS * 1024);
        const i32x4 buffer = from.buffer();
#pragma unroll
        for (int i = 0; i < LOADS; ++i) fetch_to_lds(to + i * 1024, at[i], buffer);
        from.advance(step);
    }
    __device__ __forceinline__ frag<T> operand(const char* piece, int square, int s) const {
        i16x4 half[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            half[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(
                piece + read[square % 2] + transposed_square(square, s, u)));
        return __builtin_bit_cast(frag<T>, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// WM x WN waves of MT x NT squares.
template <int MT_, int NT_, int WM_, int WN_>
struct ProductShape {
    static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, WAVES = WM * WN, THREADS = WAVES * WAVE;
    static constexpr int TILE_M = WM * MT * 32, TILE_N = WN * NT * 32;
    static constexpr int BYTES = 2 * (TILE_M + TILE_N) * PRODUCT_K * 2;
    static __device__ __forceinline__ int wave_m() { return (int)uniform(threadIdx.x / WAVE) % WM; }
    static __device__ __forceinline__ int wave_n() { return (int)uniform(threadIdx.x / WAVE) / WM; }
};

// The sums over `k`.  Every wave of the workgroup calls it; the tiles in LDS are free again after a barrier.
template <typename T, class S, class A, class B>
__device__ __forceinline__ void product(f32x16 (&c)[S::MT][S::NT], A& a, B& b, char* lds, uint32_t k) {
#pragma unroll
    for (int m = 0; m < S::MT; ++m)
#pragma unroll
        for (int n = 0; n < S::NT; ++n) c[m][n] = 0.0f;
    if (k == 0) return;
    constexpr uint32_t BUFFER = A::BYTES + B::BYTES;
    const uint32_t at = lds_address(lds);
    const int m0 = S::wave_m() * S::MT, n0 = S::wave_n() * S::NT;
    a.fetch(at, k);
    b.fetch(at + A::BYTES, k);
    uint32_t now = 0;
    for (uint32_t done = 0; done < k; done += PRODUCT_K) {
        fetched();
        const char* piece = lds + now;
        now ^= BUFFER;
        if (done + PRODUCT_K < k) {
            a.fetch(at + now, k - done - PRODUCT_K);
            b.fetch(at + now + A::BYTES, k - done - PRODUCT_K);
        }
#pragma unroll
        for (int s = 0; s < PRODUCT_K / 16; ++s) {
            frag<T> x[S::MT], y[S::NT];
#pragma unroll
            for (int m = 0; m < S::MT; ++m) x[m] = a.operand(piece, m0 + m, s);
#pragma unroll
            for (int n = 0; n < S::NT; ++n) y[n] = b.operand(piece + A::BYTES, n0 + n, s);
#pragma unroll
            for (int m = 0; m < S::MT; ++m)
#pragma unroll
                for (int n = 0; n < S::NT; ++n) c[m][n] = mfma(x[m], y[n], c[m][n]);
        }
    }
}

}  // namespace okt

#endif
