// Index arithmetic of the matrix products: where a fetch puts what, where a read finds it, and which tile is whose.
// Functions of numbers alone, so that the host can check them.
#ifndef OKT_PRODUCT_LAYOUT_H
#define OKT_PRODUCT_LAYOUT_H

#include "okt_attention_layout.h"

namespace okt {

// A piece with k contiguous: rows of 128 bytes, eight to a block of 1024, chunk c of row r at c ^ turn(r).  The rows of a square are read in
// the order in which the unit takes them: row x of B is row x; row x of A the one that makes element r of a
// lane's sixteen sums row 16 (l / 32) + r.
template <bool ORDERED>
OKT_LAYOUT_FN uint32_t kmajor_turn(uint32_t row) {
    return ORDERED ? (row % 8) ^ (row / 4 % 2) ^ (row / 16 % 2 * 4) : (row % 8) ^ (row / 8 % 2);
}
template <bool ORDERED>
OKT_LAYOUT_FN uint32_t kmajor_chunk(uint32_t lane, uint32_t block) { return lane % 8 ^ kmajor_turn<ORDERED>(block % 4 * 8 + lane / 8); }
template <bool ORDERED>
OKT_LAYOUT_FN uint32_t square_row(uint32_t x) { return ORDERED ? 16 * (x / 4 % 2) + 4 * (x / 8) + x % 4 : x; }
template <bool ORDERED>
OKT_LAYOUT_FN uint32_t kmajor_read(uint32_t lane, uint32_t s) {
    const uint32_t row = square_row<ORDERED>(lane % 32);
    return row * 128 + ((2 * s + lane / 32) ^ kmajor_turn<ORDERED>(row)) * 16;
}
constexpr uint32_t KMAJOR_SQUARE = 4096;            // bytes from 32 rows to the next

// A piece with k from row to row: blocks of eight rows by 64 columns, chunk c of row r at c ^ 4 (r / 2 % 2); the blocks of
// 64 columns one after the other, eight each.  A transposing read takes four columns a lane, of four rows for sixteen lanes.
OKT_LAYOUT_FN uint32_t transposed_chunk(uint32_t lane) { return lane % 8 ^ (lane / 16 % 2 * 4); }
template <bool ORDERED>
OKT_LAYOUT_FN uint32_t transposed_read(uint32_t lane, uint32_t half) {
    const uint32_t in = lane % 16, row = in / 4, g = lane / 16 % 2, four = in % 4;
    const uint32_t col = ORDERED ? 16 * (four % 2) + 8 * g + 4 * (four / 2) : 16 * g + 4 * four;
    return lane / 32 * 1024 + row * 128 + ((4 * half + col / 8) ^ (row / 2 % 2 * 4)) * 16 + col / 4 % 2 * 8;
}
OKT_LAYOUT_FN uint32_t transposed_square(uint32_t square, uint32_t s, uint32_t u) { return (square / 2 * 8 + 2 * s) * 1024 + u * 512; }

// Which tile of C a workgroup takes: the eight dies, to which workgroups go in turn, get consecutive tiles, four m by all n at a
// time, so that those which a die works on together share rows of both operands in its L2.
struct TilePlace { uint32_t m, n; bool there; };
OKT_LAYOUT_FN TilePlace tile_place(uint32_t group, uint32_t tiles_m, uint32_t tiles_n) {
    const uint32_t total = tiles_m * tiles_n, die = group % DIES, slot = group / DIES;
    const uint32_t from = (uint32_t)((uint64_t)total * die / DIES), to = (uint32_t)((uint64_t)total * (die + 1) / DIES);
    if (slot >= to - from) return {0, 0, false};
    constexpr uint32_t STRIP = 4;
    const uint32_t i = from + slot, strip = i / (STRIP * tiles_n), in = i % (STRIP * tiles_n);
    const uint32_t wide = tiles_m - strip * STRIP < STRIP ? tiles_m - strip * STRIP : STRIP;
    return {strip * STRIP + in % wide, in / wide, true};
}
// Workgroups of a launch whose every tile is there.
inline uint64_t tile_groups(uint64_t tiles) { return (tiles + DIES - 1) / DIES * DIES; }

}  // namespace okt

#endif
