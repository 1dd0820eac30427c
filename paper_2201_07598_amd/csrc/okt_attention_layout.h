// Who does what in the attention kernels: index arithmetic only, written so that a host
// compiler can build it too (the CPU tests check that nothing is done twice or left out).
#ifndef OKT_ATTENTION_LAYOUT_H
#define OKT_ATTENTION_LAYOUT_H

#include <stdint.h>

#ifdef __HIPCC__
#include <hip/hip_runtime.h>
#define OKT_LAYOUT_FN __host__ __device__ __forceinline__
#else
#define OKT_LAYOUT_FN static inline
#endif

namespace okt {

// The row of a 32-row tile that slot s of the A operand holds.
OKT_LAYOUT_FN constexpr uint32_t row_of_slot(uint32_t s) {
    return (s & ~31u) | ((s & 4) << 2) | ((s >> 1) & 12) | (s & 3);
}

// A divisor known on the host.  Exact for numbers below 2^30: with 2^shift >= by, mul exceeds
// 2^(30 + shift) / by by less than one, so the product by less than 2^30 2^-30.  A division by a
// number that only the kernel's arguments hold takes some twenty instructions, and a
// workgroup's place takes eight of them.
struct Divider { uint32_t by, mul, shift; };

OKT_LAYOUT_FN Divider divider(uint32_t by) {
    Divider d = {by ? by : 1, 0, 0};
    while (1u << d.shift < d.by) ++d.shift;
    d.mul = (uint32_t)(((1ull << (30 + d.shift)) + d.by - 1) / d.by);
    return d;
}
OKT_LAYOUT_FN uint32_t quotient(uint32_t n, Divider d) { return (uint32_t)((uint64_t)n * d.mul >> (30 + d.shift)); }
OKT_LAYOUT_FN uint32_t remainder(uint32_t n, Divider d) { return n - quotient(n, d) * d.by; }

// Which block of which head a workgroup takes.  A unit is what shares keys (a sequence's key
// head): `heads` heads of `blocks` blocks, the longest block first.
//   dies   Workgroups are dealt to the eight dies in turn.  A unit goes to one die, whose
//          L2 its workgroups share, and neighbouring units to different dies, so that long and
//          short sequences spread over all of them.
//   end    Under a causal mask the last `window` heads of a die are taken block by block, not
//          head by head, so that what starts last is short (2 x 16 heads x 4096 x 128: forward 157 us,
//          head by head to the end 171; backward 531 and 545, of 64 columns 323 and 344).
//   parts  A die deals its workgroups in turn over its own four parts.  Before the end, the
//          blocks of every four (or last two) are turned by another number for every head, so
//          that no part gets the first, or the empty last, block of each (32 x 16 heads x 512 x 64,
//          lengths up to 512: forward 50 us, not turned 54; backward 149 and 165).
constexpr uint32_t DIES = 8;

struct Places {
    uint32_t units, heads, blocks, window;
    Divider by_block, by_head, by_unit, by_short, by_long;     // blocks, heads, heads * blocks, units / 8, units / 8 + 1
};

OKT_LAYOUT_FN Places places(uint32_t units, uint32_t heads, uint32_t blocks, uint32_t window) {
    return {units, heads, blocks, window, divider(blocks), divider(heads), divider(heads * blocks), divider(units / DIES),
            divider(units / DIES + 1)};
}

struct Place { uint32_t unit, head, block; };

OKT_LAYOUT_FN Place place_of(uint32_t index, const Places& a) {
    const auto first = [](uint32_t die, uint32_t n) { const uint32_t more = n % DIES; return die * (n / DIES) + (die < more ? die : more); };
    const uint32_t total = a.units * a.heads * a.blocks;
    uint32_t at = first(index % DIES, total) + index / DIES;
    bool ending = false;
    if (a.window) {
        const uint32_t end = first(index % DIES + 1, total), whole = quotient(end - first(index % DIES, total), a.by_block);
        const uint32_t rows = a.window < whole ? a.window : whole, from = end - rows * a.blocks;
        ending = at >= from;
        if (ending) {
            const uint32_t k = at - from, block = k / rows;
            at = from + k % rows * a.blocks + remainder(block + a.blocks - remainder(from, a.by_block), a.by_block);   // at % blocks is `block`
        }
    }
    // units in the order of the dies' shares: number i of a die's share is unit 8 i + die
    const uint32_t run = quotient(at, a.by_unit), more = a.units % DIES, long_runs = more * (a.units / DIES + 1);
    const uint32_t die = run < long_runs ? quotient(run, a.by_long) : more + quotient(run - long_runs, a.by_short);
    const uint32_t row = quotient(at, a.by_block);
    Place p = {(run - first(die, a.units)) * DIES + die, remainder(row, a.by_head), at - row * a.blocks};
    if (!ending && a.units * a.heads % DIES == 0) {            // whole heads of every die
        const uint32_t four = p.block & ~3u, left = a.blocks - four, turn = p.unit / DIES + p.head;
        if (left >= 4) p.block = four + ((p.block + turn) & 3);
        else if (left == 2) p.block = four + ((p.block + turn) & 1);
    }
    return p;
}

// Heads that a die takes block by block at its end: as many as its L2 holds the keys and
// values of, and at least eight; none where blocks are alike.
OKT_LAYOUT_FN uint32_t window_of(bool causal, uint32_t k_len, uint32_t dim, uint32_t group) {
    if (!causal) return 0;
    const uint64_t unit_bytes = (uint64_t)k_len * dim * 4 + 1, n = (4ull << 20) / unit_bytes * group;
    return n < 8 ? 8 : n > 64 ? 64 : (uint32_t)n;
}

// Steps [first, last) of `steps`, below 2^30, that part `part` of `parts.by` takes, which are equal but
// for one; part 0 takes step 0 if there is one.
struct Part { int first, last; };
OKT_LAYOUT_FN Part part_of(int steps, uint32_t part, Divider parts) {
    const uint32_t whole = quotient((uint32_t)steps, parts), rest = (uint32_t)steps - whole * parts.by;
    const auto cut = [&](uint32_t p) { return (int)(p * whole + quotient(p * rest + parts.by - 1, parts)); };
    return {cut(part), cut(part + 1)};
}

// The most parts: enough to give every CU two workgroups, none of fewer than `least` steps.
constexpr uint32_t PART_MAX = 32;
OKT_LAYOUT_FN uint32_t parts_for(uint64_t workgroups, uint64_t steps, uint32_t least) {
    constexpr uint64_t WANTED = 512;
    if (workgroups == 0 || workgroups * 2 > WANTED) return 1;
    uint64_t n = (WANTED + workgroups - 1) / workgroups;
    if (n > steps / least) n = steps / least;
    if (n > PART_MAX) n = PART_MAX;
    return n ? (uint32_t)n : 1;
}

// How many of them are worth it: parts shorten what a workgroup does one step after the other, and cost
// another launch and their sums' way to memory and back.  `step_ns` of a step, `part_bytes` of a part
// written and read (at 6 TB/s, what such sums, which stay in the caches, were seen to take, and 0.2 us
// a part for the chain of the kernel that adds them); `launch_ns` 0 where there is that launch anyway.
constexpr uint64_t PART_LAUNCH_NS = 5000;
OKT_LAYOUT_FN uint32_t parts_worth(uint32_t most, uint64_t steps, uint64_t step_ns, uint64_t part_bytes, uint64_t launch_ns) {
    uint32_t best = 1;
    uint64_t least = steps * step_ns;
    for (uint32_t n = 2; n <= most; ++n) {
        const uint64_t ns = (steps + n - 1) / n * step_ns + n * (part_bytes / 6000 + 200) + launch_ns;
        if (ns < least) {
            least = ns;
            best = n;
        }
    }
    return best;
}

}  // namespace okt

#endif
