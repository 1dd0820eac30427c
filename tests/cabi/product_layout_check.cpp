// Host check of the matrix products' index arithmetic: what a wave's fetches put into LDS is what its reads expect there, every place
// is written once and read inside the piece, sixteen neighbouring lanes of a read hit all banks once, and every tile of C belongs to one workgroup.  Prints
// the number of cases and of violations.
#include <cstdio>
#include <set>
#include <vector>

#include "okt_product_layout.h"

using namespace okt;
static long cases = 0, bad = 0;
static void want(bool fine, const char* what, int a, int b, int c) {
    ++cases;
    if (!fine && ++bad < 20) std::printf("%s %d %d %d\n", what, a, b, c);
}

struct Chunk { int row, k; };                        // of sixteen bytes: their row (or column) and their first k (or row k)

template <bool ORDERED>
static void kmajor(int rows, int waves) {
    std::vector<Chunk> lds(rows * 8, Chunk{-1, -1});
    const int loads = rows / 8 / waves;
    for (int wave = 0; wave < waves; ++wave)
        for (int i = 0; i < loads; ++i)
            for (int lane = 0; lane < 64; ++lane) {
                Chunk& p = lds[(wave * loads + i) * 64 + lane];
                want(p.row < 0, "written twice", wave, i, lane);
                p = {(wave * loads + i) * 8 + lane / 8, (int)kmajor_chunk<ORDERED>(lane, i) * 8};
            }
    for (int square = 0; square < rows / 32; ++square)
        for (int s = 0; s < 4; ++s) {
            std::set<int> banks;
            for (int lane = 0; lane < 64; ++lane) {
                const uint32_t at = kmajor_read<ORDERED>(lane, s) + square * KMAJOR_SQUARE;
                want(at % 16 == 0 && at / 16 < lds.size(), "read outside", square, s, lane);
                const Chunk p = lds[at / 16];
                want(p.row == square * 32 + (int)square_row<ORDERED>(lane % 32) && p.k == 16 * s + lane / 32 * 8, "k-major", square, s, lane);
                if (lane % 16 == 0) banks.clear();
                want(banks.insert(at / 16 % 16).second, "k-major banks", square, s, lane);
            }
        }
}

template <bool ORDERED>
static void transposed(int columns, int waves) {
    std::vector<Chunk> lds(columns * 8, Chunk{-1, -1});       // sixteen bytes: eight columns of one k
    const int loads = columns / 8 / waves;
    for (int wave = 0; wave < waves; ++wave)
        for (int i = 0; i < loads; ++i)
            for (int lane = 0; lane < 64; ++lane) {
                const int block = wave * loads + i;
                Chunk& p = lds[block * 64 + lane];
                want(p.row < 0, "written twice", wave, i, lane);
                p = {block / 8 * 64 + (int)transposed_chunk(lane) * 8, block % 8 * 8 + lane / 8};
            }
    for (int square = 0; square < columns / 32; ++square)
        for (int s = 0; s < 4; ++s)
            for (int u = 0; u < 2; ++u) {
                uint32_t at[64];
                std::set<int> banks;
                for (int lane = 0; lane < 64; ++lane) {
                    at[lane] = transposed_read<ORDERED>(lane, square % 2) + transposed_square(square, s, u);
                    want(at[lane] % 8 == 0 && at[lane] / 16 < lds.size(), "read outside", square, s, lane);
                    if (lane % 32 == 0) banks.clear();
                    want(banks.insert(at[lane] / 8 % 32).second, "transposed banks", square, s, lane);
                }
                // what the unit hands out: lane i of sixteen gets column i of the rows that four lanes each gave
                for (int lane = 0; lane < 64; ++lane)
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t a = at[lane / 16 * 16 + 4 * j + lane % 16 / 4] + lane % 4 * 2;
                        const Chunk p = lds[a / 16];
                        want(p.row + (int)(a % 16 / 2) == square * 32 + (int)square_row<ORDERED>(lane % 32) && p.k == 16 * s + lane / 32 * 8 + 4 * u + j,
                             "transposed", square, s, lane);
                    }
            }
}

int main() {
    for (int waves : {4, 8}) {
        kmajor<false>(256, waves);
        kmajor<true>(256, waves);
        transposed<false>(256, waves);
        transposed<true>(256, waves);
    }
    kmajor<false>(128, 4);
    kmajor<true>(128, 4);
    transposed<false>(128, 4);
    transposed<true>(128, 4);
    // element r of a lane's sums is row 8 (r / 4) + 4 (l / 32) + r % 4 of A, which has to be row 16 (l / 32) + r of the square
    for (int h = 0; h < 2; ++h)
        for (int r = 0; r < 16; ++r) want((int)square_row<true>(8 * (r / 4) + 4 * h + r % 4) == 16 * h + r, "order", h, r, 0);
    for (uint32_t m : {1u, 2u, 3u, 4u, 5u, 7u, 8u, 16u, 119u, 500u})
        for (uint32_t n : {0u, 1u, 2u, 3u, 9u, 32u, 64u}) {
            std::set<uint64_t> seen;
            for (uint64_t g = 0; g < tile_groups((uint64_t)m * n) + 24; ++g) {
                const TilePlace t = tile_place((uint32_t)g, m, n);
                if (!t.there) continue;
                want(t.m < m && t.n < n && g < tile_groups((uint64_t)m * n), "tile", m, n, (int)g);
                want(seen.insert((uint64_t)t.m << 32 | t.n).second, "tile twice", m, n, (int)g);
            }
            want(seen.size() == (uint64_t)m * n, "tiles", m, n, (int)seen.size());
        }
    std::printf("%ld cases, %ld violations\n", cases, bad);
    return bad ? 1 : 0;
}
