// Host check of the attention kernels' index arithmetic: every block of every head is taken by one
// workgroup, whatever the numbers; the parts of an axis cover it once, part 0 with its
// beginning; the slots of a tile are a permutation of its rows.  Prints the number of violations.
#include <cstdio>
#include <set>
#include <tuple>

#include "okt_attention_layout.h"

int main() {
    long bad = 0, cases = 0;
    for (uint32_t units : {1u, 2u, 3u, 5u, 7u, 8u, 9u, 15u, 16u, 25u, 32u, 64u, 100u, 512u})
        for (uint32_t heads : {1u, 2u, 3u, 4u, 7u})
            for (uint32_t blocks : {1u, 2u, 3u, 4u, 5u, 8u, 31u, 33u})
                for (uint32_t window : {0u, 1u, 8u, 64u}) {
                    std::set<std::tuple<uint32_t, uint32_t, uint32_t>> seen;
                    const uint32_t total = units * heads * blocks;
                    const okt::Places places = okt::places(units, heads, blocks, window);
                    for (uint32_t i = 0; i < total; ++i) {
                        const okt::Place p = okt::place_of(i, places);
                        if (p.unit >= units || p.head >= heads || p.block >= blocks) ++bad;
                        seen.insert({p.unit, p.head, p.block});
                    }
                    if (seen.size() != total) ++bad;
                    ++cases;
                }
    const int many[] = {1000, 65537, 12345678, (1 << 30) - 1};
    for (int n = 0; n < 204; ++n) {
        const int steps = n < 200 ? n : many[n - 200];
        for (uint32_t parts = 1; parts <= okt::PART_MAX; ++parts) {
            int at = 0;
            for (uint32_t p = 0; p < parts; ++p) {
                const okt::Part part = okt::part_of(steps, p, okt::divider(parts));
                if (part.first != at || part.last < part.first) ++bad;
                if (p == 0 && steps && part.last == 0) ++bad;
                at = part.last;
            }
            if (at != steps) ++bad;
            ++cases;
        }
    }
    for (uint64_t groups = 0; groups < 2000; groups += 7)
        for (uint64_t steps = 0; steps < 300; steps += 11)
            for (uint32_t least : {1u, 2u, 4u}) {
                const uint32_t n = okt::parts_for(groups, steps, least);
                if (n < 1 || n > okt::PART_MAX || (n > 1 && n * (uint64_t)least > steps)) ++bad;
                // never slower by its own reckoning than no parts, and no parts where a launch costs more than all steps
                for (uint64_t bytes : {(uint64_t)0, (uint64_t)1 << 20, (uint64_t)1 << 50}) {
                    const uint32_t worth = okt::parts_worth(n, steps, 750, bytes, okt::PART_LAUNCH_NS);
                    if (worth < 1 || worth > n || (bytes >> 50 && worth > 1) || (steps * 750 <= okt::PART_LAUNCH_NS && worth > 1)) ++bad;
                }
                ++cases;
            }
    for (uint32_t by = 1; by < (1u << 30); by = by < 5000 ? by + 1 : by + by / 7 + 1) {
        const okt::Divider d = okt::divider(by);
        for (uint32_t m : {0u, 1u, 2u, 3u, 1000u, ((1u << 30) - 1) / by, ((1u << 30) - 1) / by / 2})
            for (int64_t off : {(int64_t)-1, (int64_t)0, (int64_t)1, (int64_t)(by / 2)}) {
                const int64_t n = (int64_t)m * by + off;
                if (n < 0 || n >= (1ll << 30)) continue;
                if (okt::quotient((uint32_t)n, d) != n / by || okt::remainder((uint32_t)n, d) != n % by) ++bad;
                ++cases;
            }
    }
    uint64_t rows = 0;
    for (uint32_t s = 0; s < 32; ++s) rows |= 1ull << okt::row_of_slot(s);
    if (rows != 0xffffffffull) ++bad;
    for (uint32_t s = 0; s < 128; ++s) {
        // element r of lane half h of a product's tile is slot 8 (r / 4) + 4 h + r % 4, and has to be row 16 h + r
        const uint32_t h = s >> 2 & 1, r = (s >> 3 & 3) * 4 + (s & 3);
        if (okt::row_of_slot(s) != (s & ~31u) + 16 * h + r) ++bad;
    }
    std::printf("%ld cases, %ld violations\n", cases, bad);
    return bad != 0;
}
