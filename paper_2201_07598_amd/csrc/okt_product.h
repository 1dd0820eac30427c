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
    OperandSource from;
    uint32_t at[LOADS], read[4];

    // Which sixteen-byte chunk of its row a lane fetches with fetch i of its wave's; blocks repeat after four.
    static __device__ __forceinline__ uint32_t chunk(int i) {
        return kmajor_chunk<ORDERED>(threadIdx.x % WAVE, LOADS % 4 == 0 ? i : threadIdx.x / WAVE * LOADS + i);
    }

    // `end`: of the tensor's last row
    __device__ __forceinline__ KMajor(const T* tile, const T* end, uint32_t row_bytes) {
        const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
        from = {(uint64_t)tile, (uint64_t)end - (uint64_t)tile};
#pragma unroll
        for (int i = 0; i < LOADS; ++i) at[i] = ((wave * LOADS + i) * 8 + lane / 8) * row_bytes + chunk(i) * 16;
#pragma unroll
        for (uint32_t s = 0; s < 4; ++s) read[s] = kmajor_read<ORDERED>(lane, s);
    }
    // Fetch i of the wave's of a piece of which the tensor has `there` k.
    __device__ __forceinline__ void fetch(int i, uint32_t lds, i32x4 buffer, uint32_t there) const {
        const uint32_t to = lds + uniform(threadIdx.x / WAVE) * (LOADS * 1024) + i * 1024;
        fetch_to_lds(to, there >= PRODUCT_K || chunk(i) * 8 < there ? at[i] : OUTSIDE, buffer);
    }
    __device__ __forceinline__ void advance() { from.advance(PRODUCT_K * 2); }
    __device__ __forceinline__ frag<T> operand(const char* piece, int square, int s) const {
        return *reinterpret_cast<const frag<T>*>(piece + read[s] + square * KMAJOR_SQUARE);
    }
};

// The same with rows from a table in LDS, all within 2^31 bytes of the tensor's first; zeros for those that are NO_ROW.
constexpr uint32_t NO_ROW = 0xffffffffu;
template <typename T, int ROWS, int WAVES>
struct ListedRows : KMajor<T, ROWS, WAVES, false> {
    typedef KMajor<T, ROWS, WAVES, false> Base;
    __device__ __forceinline__ ListedRows(const T* tensor, const T* end, uint32_t row_bytes, const uint32_t* rows) : Base(tensor, end, 0) {
        const uint32_t lane = threadIdx.x % WAVE, wave = threadIdx.x / WAVE;
#pragma unroll
        for (int i = 0; i < Base::LOADS; ++i) {
            const uint32_t row = rows[(wave * Base::LOADS + i) * 8 + lane / 8];
            this->at[i] = row == NO_ROW ? OUTSIDE : row * row_bytes + Base::chunk(i) * 16;
        }
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
    __device__ __forceinline__ void fetch(int i, uint32_t lds, i32x4 buffer, uint32_t) const {
        fetch_to_lds(lds + uniform(threadIdx.x / WAVE) * (LOADS * 1024) + i * 1024, at[i], buffer);
    }
    __device__ __forceinline__ void advance() { from.advance(step); }
    __device__ __forceinline__ frag<T> operand(const char* piece, int square, int s) const {
        i16x4 half[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            half[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(
                piece + read[square % 2] + transposed_square(square, s, u)));
        return __builtin_bit_cast(frag<T>, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

template <class S>
__device__ __forceinline__ void clear(f32x16 (&c)[S::MT][S::NT]) {
#pragma unroll
    for (int m = 0; m < S::MT; ++m)
#pragma unroll
        for (int n = 0; n < S::NT; ++n) c[m][n] = 0.0f;
}

// WM x WN waves of MT x NT squares, and buffers in LDS for STAGES pieces: one is worked on, the others are on their way.
template <int MT_, int NT_, int WM_, int WN_, int STAGES_>
struct ProductShape {
    static constexpr int MT = MT_, NT = NT_, WM = WM_, WN = WN_, STAGES = STAGES_, WAVES = WM * WN, THREADS = WAVES * WAVE;
    static constexpr int TILE_M = WM * MT * 32, TILE_N = WN * NT * 32;
    static constexpr int BYTES = STAGES * (TILE_M + TILE_N) * PRODUCT_K * 2;
    static __device__ __forceinline__ int wave_m() { return (int)uniform(threadIdx.x / WAVE) % WM; }
    static __device__ __forceinline__ int wave_n() { return (int)uniform(threadIdx.x / WAVE) / WM; }
};

// Waits for this wave's fetches into LDS but the last LEFT, and for its reads from there, then for the other waves.
template <int LEFT>
__device__ __forceinline__ void handed_over() {
    static_assert(LEFT < 64, "the counter has six bits");
    __builtin_amdgcn_s_waitcnt((LEFT & 15) | (LEFT >> 4) << 14 | 0x0070);      // vmcnt(LEFT), lgkmcnt(0)
    __syncthreads();
}

// The sums over `k`: begin() sends out the first fetches, run() does the rest.  Every wave of the workgroup calls both; the tiles in LDS have to be
// free at begin() and are free again after run(), so the next tile's begin() can stand before this one's sums are stored.
//
// A piece is four steps of sixteen k.  While a step's products run, the wave reads the next step's operands from LDS, a few between every
// NT products, and the barrier that hands over the next piece stands before the last step, whose operands are in registers by then: so the
// products of that step cover the first reads of the next piece and the first fetches of the one after it.  Fetches go out one by one
// between products, half of a piece's in that step and half in the next one (8192 x 128000 x 4096: 6.5 ms; all together, which holds the wave
// up for a thousand cycles, 7.2; all in the last step 6.7, over three steps 6.6).  Two waves a SIMD, 128 x 64 each: one of 128 x 128
// reads a quarter less from LDS and takes 6.7.
template <typename T, class S, class A, class B, bool AGAIN = false>
struct Product {
    static constexpr uint32_t BUFFER = A::BYTES + B::BYTES;
    static constexpr int LOADS = A::LOADS + B::LOADS, LEFT = (S::STAGES - 2) * LOADS;
    static_assert(S::NT <= S::MT, "a group reads one operand of each side");
    A a;
    B b;
    uint32_t k, at;
    i32x4 buffer_a, buffer_b;
    uint32_t ahead, there;                                           // k before the piece that is fetched, and in and behind it
    OperandSource again_a, again_b;                                  // AGAIN: where both sides go on from k = again on
    uint32_t again = 0;                                              // (0: they do not)

    __device__ __forceinline__ void fetch(int i, uint32_t to) const {
        if (i < A::LOADS) a.fetch(i, at + to, buffer_a, there);
        else if (i < LOADS) b.fetch(i - A::LOADS, at + to + A::BYTES, buffer_b, there);
    }
    __device__ __forceinline__ void next_piece() {
        there = ahead < k ? k - ahead : 0;
        if (AGAIN && again && ahead == again) {
            a.from = again_a;
            b.from = again_b;
        }
        buffer_a = a.from.buffer();
        buffer_b = b.from.buffer();
        if (there == 0) buffer_a[2] = buffer_b[2] = 0;               // past the end nothing is read
        a.advance();
        b.advance();
        ahead += PRODUCT_K;
    }
    __device__ __forceinline__ Product(const A& a_, const B& b_, uint32_t k_, const char* lds) : a(a_), b(b_), k(uniform(k_)), at(lds_address(lds)) {}

    __device__ __forceinline__ void begin() {
        ahead = 0;
        if (k == 0) return;
#pragma unroll
        for (int p = 0; p < S::STAGES - 1; ++p) {
            next_piece();
#pragma unroll
            for (int i = 0; i < LOADS; ++i) fetch(i, p * BUFFER);
        }
    }

    // Adds to c.
    __device__ __forceinline__ void run(f32x16 (&c)[S::MT][S::NT], const char* lds) {
        if (k == 0) return;
        constexpr int STEPS = PRODUCT_K / 16, EARLY = LOADS / 2, LATE = LOADS - EARLY;       // fetches in the last step, in the first
        constexpr int EACH = ((EARLY > LATE ? EARLY : LATE) + S::MT - 1) / S::MT;
        const int m0 = S::wave_m() * S::MT, n0 = S::wave_n() * S::NT;
        frag<T> x[2][S::MT], y[2][S::NT];
        // the operands of a step that a group of products covers
        const auto read = [&](int set, int m, const char* piece, int s) {
            x[set][m] = a.operand(piece, m0 + m, s);
            if (m < S::NT) y[set][m] = b.operand(piece + A::BYTES, n0 + m, s);
        };
        handed_over<LEFT>();
        next_piece();
        uint32_t now = 0, filled = (S::STAGES - 1) * BUFFER;         // the buffer that is worked on, and the one that is filled
#pragma unroll
        for (int i = 0; i < EARLY; ++i) fetch(i, filled);
#pragma unroll
        for (int m = 0; m < S::MT; ++m) read(0, m, lds, 0);
        for (uint32_t done = PRODUCT_K; ; done += PRODUCT_K) {       // k up to the end of this piece
            const uint32_t next = now + BUFFER < S::BYTES ? now + BUFFER : 0;
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                if (s == STEPS - 1) {
                    handed_over<LEFT>();
                    next_piece();
                    filled = now;
                }
                const char* piece = lds + (s == STEPS - 1 ? next : now);
#pragma unroll
                for (int m = 0; m < S::MT; ++m) {
                    __builtin_amdgcn_sched_barrier(0);
                    read((s + 1) % 2, m, piece, (s + 1) % STEPS);
#pragma unroll
                    for (int i = 0; i < EACH; ++i) {
                        if (s == 0 && m * EACH + i < LATE) fetch(EARLY + m * EACH + i, filled);
                        if (s == STEPS - 1 && m * EACH + i < EARLY) fetch(m * EACH + i, filled);
                    }
#pragma unroll
                    for (int n = 0; n < S::NT; ++n) c[m][n] = mfma(x[s % 2][m], y[s % 2][n], c[m][n]);
                }
            }
            now = next;
            if (done >= k) break;
        }
        __builtin_amdgcn_sched_barrier(0);
        handed_over<0>();                                            // nothing is on its way into LDS any more
    }
};

}  // namespace okt

#endif
