// What the attention kernels share: the matrix unit's tiles, the tiles of rows in LDS, the
// dropout mask's shares, and the host's checks.
//
// Products are 32 x 32 x 16 steps of the matrix unit, C += A B with 16-bit inputs:
//   A  lane l holds row l % 32, columns 8 (l / 32) .. + 7
//   B  lane l holds column l % 32, rows 8 (l / 32) .. + 7
//   C  lane l holds column l % 32, element r is row 8 (r / 4) + 4 (l / 32) + r % 4
// Rows of A are kept in LDS in the order that makes element r of C the row 16 (l / 32) + r
// of the tile (row_of_slot): then elements 8t .. 8t + 7 of C are, as they lie, the B operand of
// step t of a product that sums over those rows.  Scores therefore go from the
// first product through the softmax into the second one without leaving their registers.
#ifndef OKT_ATTENTION_H
#define OKT_ATTENTION_H

#include "okt_attention_layout.h"
#include "okt_element.h"
#include "okt_random.h"

namespace okt {

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
typedef short i16x8 __attribute__((ext_vector_type(8)));

template <typename T> using frag = typename Eight<T>::vec;

__device__ __forceinline__ f32x16 mfma(frag<__bf16> a, frag<__bf16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma(frag<_Float16> a, frag<_Float16> b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// Eight neighbouring elements of a C tile as a B operand: rounded to the tensors' type, and if FINE a second operand
// of what the rounding left off, so that the product is that of 16 (fp16: 22) bits.  The rounding is what the matrix units'
// rate costs: products of fp32 operands run at a sixteenth of it.
template <typename T, bool FINE>
struct Operand {
    frag<T> rounded, rest;
    __device__ __forceinline__ Operand(const f32x16& c, int t) {
        f32x8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = c[8 * t + i];
        rounded = __builtin_convertvector(v, frag<T>);
        if (FINE) rest = __builtin_convertvector(v - __builtin_convertvector(rounded, f32x8), frag<T>);
    }
};

template <typename T, bool FINE>
__device__ __forceinline__ f32x16 mfma(frag<T> a, const Operand<T, FINE>& b, f32x16 c) {
    if (FINE) c = mfma(a, b.rest, c);
    return mfma(a, b.rounded, c);
}

// Probabilities are operands of the second products in the tensors' type.  bf16 has the exponents of fp32; fp16 ends
// at 2^-24, below which long flat rows have much of their weight, so there they are taken times a power of two
// that is divided out of the sums: the forward pass holds a row's largest between 2^7 and 2^15 (fp16 ends at 2^16),
// the keys' kernel takes 2^12 p.
template <typename T> struct Raised { static constexpr float forward = 0.0f, keys = 0.0f, keys_factor = 1.0f; };
template <> struct Raised<_Float16> { static constexpr float forward = 7.0f, keys = 12.0f, keys_factor = 4096.0f; };

// ------------------------------------------------------------------ tiles of rows in LDS

typedef int i32x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t OUTSIDE = 0xffff0000u;     // an offset that no buffer reaches

// 16 bytes a lane from `buffer` at its byte offset to LDS, lane after lane from `lds` on; 0
// where the offset is outside the buffer.  Written out because the compiler, which cannot
// tell the tile that is being filled from the one that is read, would wait for it before the next read
// of LDS; fetched() waits where it has to be.
__device__ __forceinline__ void fetch_to_lds(uint32_t lds, uint32_t offset, i32x4 buffer) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :: "s"(lds), "v"(offset), "s"(buffer) : "m0", "memory");
}

__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void*)p;
}

// ROWS rows of DIM elements, rows in the order of slots, as blocks of sixteen slots by four
// chunks of eight elements: 1024 bytes, what one fetch of a wave fills, four lanes to 64 bytes of
// a row.  In a block chunk c of slot s lies at 64 s + 16 (c ^ s / 4).  Sixteen neighbouring
// slots then read one chunk from all banks (A operands, row by row), and so do the four
// slots by four chunks of a transposing read; and what a lane adds for another tile, step or
// column is a constant, so a kernel keeps four offsets for all its reads.
struct TileReads {
    uint32_t rows[2], columns[2];                   // of even and odd steps; of the two halves of a step
};

template <typename T, int DIM, int ROWS, int THREADS>
struct RowTile {
    static constexpr int ACROSS = DIM / 32;                     // blocks of sixteen slots
    static constexpr int BYTES = ROWS * DIM * 2;
    static constexpr int LOADS = BYTES / 1024 / (THREADS / WAVE);   // of a wave

    static __device__ __forceinline__ uint32_t fetched_slot(int i) {
        const uint32_t lane = threadIdx.x % WAVE, block = i * (THREADS / WAVE) + threadIdx.x / WAVE;
        return block / ACROSS * 16 + lane / 4;
    }

    // What a thread fetches of every tile, in bytes from the tile's first row; places past
    // head_dim lie beyond any tensor and read as 0.
    struct Places {
        uint32_t at[LOADS];
        __device__ __forceinline__ Places(uint32_t row_bytes, uint32_t head_dim) {
#pragma unroll
            for (int i = 0; i < LOADS; ++i) {
                const uint32_t block = i * (THREADS / WAVE) + threadIdx.x / WAVE, lane = threadIdx.x % WAVE;
                const uint32_t chunk = block % ACROSS * 4 + (lane % 4 ^ lane / 16);
                at[i] = DIM == (int)head_dim || chunk * 8 < head_dim ? row_of_slot(fetched_slot(i)) * row_bytes + chunk * 16 : OUTSIDE;
            }
        }
    };

    // Tiles of a tensor one after the other, straight into LDS.  The buffer's bounds end with the
    // last row, so that rows past it arrive as zeros whatever lies there.
    struct Stream {
        uint64_t at, left, step;                    // of the next tile: its address, bytes to the tensor's end
        __device__ __forceinline__ Stream(const T* base, uint32_t row_bytes, int first, int count, uint32_t head_dim)
            : at((uint64_t)base + (uint64_t)first * row_bytes), left((uint64_t)(count - first - 1) * row_bytes + head_dim * 2),
              step((uint64_t)ROWS * row_bytes) {}
        // `before`: how many rows at the tile's beginning are not looked at, either
        __device__ __forceinline__ void fetch(uint32_t tile, const Places& p, int before = 0) {
            const uint32_t wave = uniform(threadIdx.x / WAVE);
            const i32x4 buffer = {(int)uniform((uint32_t)at), (int)uniform((uint32_t)(at >> 32)),
                                  (int)uniform(left < OUTSIDE ? (uint32_t)left : OUTSIDE), 0x00020000};
            if (before <= 0) {
#pragma unroll
                for (int i = 0; i < LOADS; ++i) fetch_to_lds(tile + (i * (THREADS / WAVE) + wave) * 1024, p.at[i], buffer);
            } else {
#pragma unroll
                for (int i = 0; i < LOADS; ++i)
                    fetch_to_lds(tile + (i * (THREADS / WAVE) + wave) * 1024,
                                 (int)row_of_slot(fetched_slot(i)) < before ? OUTSIDE : p.at[i], buffer);
            }
            at += step;
            left = left > step ? left - step : 0;
        }
    };

    static __device__ __forceinline__ TileReads reads() {
        const uint32_t lane = threadIdx.x % WAVE, in = lane % 16;
        TileReads r;
#pragma unroll
        for (uint32_t odd = 0; odd < 2; ++odd) {
            const uint32_t c = 2 * odd + lane / 32;
            r.rows[odd] = lane % 32 / 16 * (ACROSS * 1024) + in * 64 + (c ^ in / 4) * 16;
        }
#pragma unroll
        for (uint32_t u = 0; u < 2; ++u) {
            const uint32_t c = 2 * (lane / 16 % 2) + in % 4 / 2;
            r.columns[u] = (8 * u + 4 * (lane / 32) + in / 4) * 64 + (c ^ (2 * u + lane / 32)) * 16 + in % 2 * 8;
        }
        return r;
    }

    // A operand: rows of the 32-row tile at slot0, columns 16 step .. + 15.
    static __device__ __forceinline__ frag<T> rows(const char* tile, const TileReads& r, uint32_t slot0, int step) {
        return *reinterpret_cast<const frag<T>*>(tile + r.rows[step % 2] + slot0 / 16 * (ACROSS * 1024) + step / 2 * 1024);
    }

    // A operand of the transpose: rows = columns 32 dt .. + 31 of the tile, columns = the
    // sixteen rows of step t of its 32-row tile at slot0.
    static __device__ __forceinline__ frag<T> columns(const char* tile, const TileReads& r, uint32_t slot0, int dt, int t) {
        i16x4 half[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
            half[u] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4*)(
                tile + r.columns[u] + (slot0 / 16 + t) * (ACROSS * 1024) + dt * 1024));
        return __builtin_bit_cast(frag<T>, __builtin_shufflevector(half[0], half[1], 0, 1, 2, 3, 4, 5, 6, 7));
    }
};

// 16 bytes a lane of what lies between `from` and `to`, straight into LDS by one wave; zeros past `to`.
__device__ __forceinline__ void fetch_line(uint32_t lds, const void* from, const void* to) {
    const uint64_t at = (uint64_t)from, bytes = (uint64_t)to - at;
    const i32x4 buffer = {(int)uniform((uint32_t)at), (int)uniform((uint32_t)(at >> 32)),
                          (int)(bytes < OUTSIDE ? uniform((uint32_t)bytes) : OUTSIDE), 0x00020000};
    fetch_to_lds(lds, threadIdx.x % WAVE * 16, buffer);
}

// Waits for this wave's fetches into LDS, then for the others.
__device__ __forceinline__ void fetched() {
    __builtin_amdgcn_s_waitcnt(0x0F70);           // vmcnt(0)
    __syncthreads();
}

// B operands straight from memory: lane's row, for each step columns 16 step + 8 (l / 32) .. + 7.
template <int DIM, typename T>
__device__ __forceinline__ void row_operands(frag<T> (&v)[DIM / 16], const T* row, uint32_t head_dim) {
    const uint32_t from = 8 * (threadIdx.x % WAVE / 32);
    if (head_dim == DIM) {
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) v[s] = *reinterpret_cast<const frag<T>*>(row + from + 16 * s);
    } else {
#pragma unroll
        for (int s = 0; s < DIM / 16; ++s) {
            v[s] = frag<T>{};
            if (from + 16 * s < head_dim) v[s] = *reinterpret_cast<const frag<T>*>(row + from + 16 * s);
        }
    }
}

// Between a lane and the one 32 away.
__device__ __forceinline__ float max_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_halves(float v) {
    const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Stores a transposed C tile column by column: lane's row, columns 32 dt + 8a + 4 (l / 32) .. + 3.
template <typename T, int TILES>
__device__ __forceinline__ void store_row(T* row, const f32x16 (&c)[TILES], float scale, uint32_t head_dim) {
    typedef T four __attribute__((ext_vector_type(4)));
    typedef float f32x4 __attribute__((ext_vector_type(4)));
    const uint32_t from = 4 * (threadIdx.x % WAVE / 32);
    const auto piece = [&](int dt, int a) {
        const f32x4 v = {c[dt][4 * a] * scale, c[dt][4 * a + 1] * scale, c[dt][4 * a + 2] * scale, c[dt][4 * a + 3] * scale};
        *reinterpret_cast<four*>(row + from + 32 * dt + 8 * a) = __builtin_convertvector(v, four);
    };
    if (head_dim == TILES * 32) {
#pragma unroll
        for (int n = 0; n < TILES * 4; ++n) piece(n / 4, n % 4);
    } else {
#pragma unroll
        for (int n = 0; n < TILES * 4; ++n)
            if (from + 8 * n < head_dim) piece(n / 4, n % 4);
    }
}

// ------------------------------------------------------------------ the dropout mask
//
// A block of the random field is two queries by four keys, so that lanes which hold a
// query's keys and lanes which hold a key's queries both share blocks with neighbours
// and none is drawn twice in a pass over a tile.

// The row of its tile that a lane takes as its own: even rows in one row of sixteen lanes, odd
// rows in the next, so that those which share blocks can swap words in one instruction.
__device__ __forceinline__ uint32_t row_of_lane() { return threadIdx.x % 16 * 2 + threadIdx.x / 16 % 2; }

// Even rows of sixteen lanes get `a` of their own and of the lanes after them, odd ones `b` of the
// lanes before them and of their own.
__device__ __forceinline__ void swap_sixteens(uint32_t& a, uint32_t& b) {
    const auto r = __builtin_amdgcn_permlane16_swap(a, b, false, false);
    a = r[0];
    b = r[1];
}

// The same between neighbouring lanes.
__device__ __forceinline__ void swap_neighbours(uint32_t& a, uint32_t& b) {
    const bool odd = threadIdx.x & 1;
    const uint32_t got = (uint32_t)__builtin_amdgcn_mov_dpp((int)(odd ? a : b), 0xB1, 0xf, 0xf, true);
    a = odd ? got : a;
    b = odd ? b : got;
}

// Whether element r is kept, of sixteen whose values lie two to a word.
__device__ __forceinline__ bool kept_element(const uint32_t (&w)[8], int r, uint32_t bar) {
    return r & 1 ? w[r / 2] < bar << 16 : (uint16_t)w[r / 2] < (uint16_t)bar;       // bar is below 65536 here
}

// Lane = query, element r = key 16 (l / 32) + r of the tile that begins at key0 (a multiple of 32).  The
// two lanes of a pair of queries draw two of the four blocks each and swap the halves that
// are the other's.
__device__ __forceinline__ void kept_keys(uint32_t (&w)[8], uint32_t query, uint32_t key0, uint32_t plane, RandomKey key,
                                          uint32_t site) {
    const uint32_t lane = threadIdx.x % WAVE;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const RandomBlock b = random_block(key, key0 / 4 + 4 * (lane / 32) + 2 * (lane / 16 % 2) + i, query / 2, plane, site);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
            w[2 * i + p] = __builtin_amdgcn_perm(b.w[2 * p + 1], b.w[2 * p], 0x05040100u);          // low halves
            w[2 * i + p + 4] = __builtin_amdgcn_perm(b.w[2 * p + 1], b.w[2 * p], 0x07060302u);      // high halves
        }
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) swap_sixteens(w[p], w[p + 4]);
}

// Lane = key, element r = query 16 (l / 32) + r of the tile that begins at query0 (a multiple of 32):
// w[p] is the word of queries 2p and 2p + 1.  Each of the four lanes that hold the keys of a
// block draws two of the eight, and a 4 x 4 transpose hands every lane its key's words.
__device__ __forceinline__ void kept_queries(uint32_t (&w)[8], uint32_t key_index, uint32_t query0, uint32_t plane,
                                             RandomKey key, uint32_t site) {
    const uint32_t lane = threadIdx.x % WAVE;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        RandomBlock b = random_block(key, key_index / 4, query0 / 2 + 8 * (lane / 32) + 4 * i + row_of_lane() % 4, plane, site);
        swap_sixteens(b.w[0], b.w[1]);
        swap_sixteens(b.w[2], b.w[3]);
        swap_neighbours(b.w[0], b.w[2]);
        swap_neighbours(b.w[1], b.w[3]);
#pragma unroll
        for (int p = 0; p < 4; ++p) w[4 * i + p] = b.w[p];
    }
}

// ------------------------------------------------------------------ work split over the long axis
//
// A workgroup owns a block of rows and passes over the other axis; where blocks are few, each
// is dealt to several workgroups that pass over a part each and leave fp32 sums in the
// workspace, which another launch joins in a fixed order.

// Stores a transposed C tile as fp32: lane's row of DIM floats.
template <int TILES>
__device__ __forceinline__ void store_partial(float* row, const f32x16 (&c)[TILES], float scale) {
#pragma unroll
    for (int dt = 0; dt < TILES; ++dt)
#pragma unroll
        for (int a = 0; a < 4; ++a)
            *reinterpret_cast<float4*>(row + 32 * dt + 8 * a + 4 * (threadIdx.x % WAVE / 32)) = make_float4(
                c[dt][4 * a] * scale, c[dt][4 * a + 1] * scale, c[dt][4 * a + 2] * scale, c[dt][4 * a + 3] * scale);
}

// The launches of a call and the parts of the workspace, from its sizes alone.
struct AttentionPlan {
    uint32_t dim;                                   // 64 or 128
    uint32_t forward_parts, query_parts, key_parts;
    uint64_t forward_groups, query_groups, key_groups;      // workgroups of each kernel
    bool packed;                                    // forward: see its kernel
    bool fine;                                      // second products from both parts of their operands
    size_t rows_at;                                 // backward: two numbers of every row
    size_t dq_at, dkv_at;                           // backward: partial sums
    size_t forward_bytes, bytes;                    // of the workspace, forward and backward
};
AttentionPlan attention_plan(uint32_t batch, uint32_t heads, uint32_t kv_heads, uint32_t q_len, uint32_t k_len, uint32_t head_dim,
                             bool drop);

constexpr uint32_t ATTENTION_QUERIES = 128;         // a workgroup of the forward and the queries' kernels
constexpr uint32_t ATTENTION_KEYS = 64;             // keys that pass by it together

// The keys' kernel: four waves are GROUPS groups of 32 keys, each HALVES times, once for every
// part of a tile of TILE queries.
template <int DIM> struct KeysShape;
template <> struct KeysShape<64> { static constexpr int GROUPS = 4, HALVES = 1, TILE = 64; };
template <> struct KeysShape<128> { static constexpr int GROUPS = 2, HALVES = 2, TILE = 128; };

// ------------------------------------------------------------------ arguments

struct Strides { uint64_t batch, row, head; };

struct AttentionArgs {
    uint32_t batch, heads, kv_heads, group, q_len, k_len, head_dim, site;
    Divider by_kv;                               // kv_heads
    bool causal;
    float scale, scale_log2;                     // scale * log2 e: scores are taken to base 2
    DropoutRule drop;
    const uint64_t* seed;
    const int32_t *q_lens, *k_lens;
    Strides q, k, v, o, d_o, dq, dk, dv;
};

// Checks the arguments of a direction and fills the kernels'; false if refused.
bool attention_args(const okt_attention* op, bool backward, AttentionArgs& a);

// Workgroups of 256 threads that a launch can have: it counts work-items in 32 bits.
constexpr uint64_t LAUNCH_GROUPS = (1ull << 24) - 1;

// Whether two tensors begin in the same place: their first vectors share an element.
inline bool same_place(const void* a, const void* b, uint32_t head_dim) { return a && b && overlap(a, head_dim * 2, b, head_dim * 2); }

// Lengths of a sequence, held to the tensors'.
__device__ __forceinline__ int sequence_length(const int32_t* lens, uint32_t b, uint32_t most) {
    if (!lens) return (int)most;
    const int n = lens[b];
    return n < 0 ? 0 : n > (int)most ? (int)most : n;
}

}  // namespace okt

#endif
