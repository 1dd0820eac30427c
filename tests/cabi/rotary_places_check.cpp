// Host check of which places the rotation writes, without a GPU: thousands of small layouts, of which every element is listed one by one.
//   self    an output is refused exactly where two of its heads share an element
//   pairs   with strides alike, outputs are refused exactly where they share an element with one another or with an input that lies elsewhere
//   far     strides and sizes at the ends of what the header allows: refused or launched, and soon
// Pointers are made up and never read.  Prints the number of cases and of violations.
#include <chrono>
#include <cstdio>
#include <cstring>
#include <random>
#include <set>

#include "launch_stub.h"
#include "okt.h"

static long cases = 0, bad = 0, refused = 0;
static char* at(uint64_t n) { return (char*)(n << 44); }

struct Layout { uint32_t batch, length, heads, dim; uint64_t s[3]; };

static std::set<int64_t> elements(const Layout& t, int64_t from, bool* twice = nullptr) {
    std::set<int64_t> out;
    for (uint32_t b = 0; b < t.batch; ++b)
        for (uint32_t i = 0; i < t.length; ++i)
            for (uint32_t h = 0; h < t.heads; ++h)
                for (uint32_t e = 0; e < t.dim; ++e)
                    if (!out.insert(from + (int64_t)(b * t.s[0] + i * t.s[1] + h * t.s[2] + e)).second && twice) *twice = true;
    return out;
}
static bool meet(const std::set<int64_t>& a, const std::set<int64_t>& b) {
    for (int64_t x : a)
        if (b.count(x)) return true;
    return false;
}

static okt_norm_rotary op_of(uint32_t batch, uint32_t length, uint32_t heads, uint32_t kv_heads, uint32_t dim) {
    okt_norm_rotary op;
    std::memset(&op, 0, sizeof op);
    op.batch = batch;
    op.length = length;
    op.heads = heads;
    op.kv_heads = kv_heads;
    op.head_dim = op.rot_dim = dim;
    op.dtype = OKT_BF16;
    op.kind = OKT_NORM_RMS;
    op.axes = 1;
    op.d_inv_freq = (const float*)at(9);
    return op;
}
static void put(uint64_t (&to)[3], const uint64_t (&s)[3]) { std::memcpy(to, s, sizeof to); }

static void expect(int status, bool accepted, const char* what, const Layout& t, int64_t apart) {
    ++cases;
    refused += !accepted;
    const bool launched = !g_launched.empty();
    g_launched.clear();
    if (status == (accepted ? OKT_OK : OKT_ERR_INVALID_ARG) && launched == accepted) return;
    if (++bad < 20)
        std::printf("%s: %u x %u x %u x %u, strides %llu %llu %llu, apart %lld: status %d where %s\n", what, t.batch, t.length, t.heads, t.dim,
                    (unsigned long long)t.s[0], (unsigned long long)t.s[1], (unsigned long long)t.s[2], (long long)apart, status, accepted ? "it is fine" : "memory is shared");
}

static std::mt19937 rng(1);
static uint32_t pick(uint32_t n) { return rng() % n; }

static Layout random_layout() {
    Layout t = {1 + pick(3), 1 + pick(4), 1 + pick(4), 8u * (1 + pick(3)), {}};
    for (uint64_t& s : t.s) s = pick(5) == 0 ? 8 * pick(60) : (pick(2) ? t.dim : 8) * pick(14) + (pick(8) == 0 ? pick(8) : 0);
    if (pick(2)) {                                                   // as they mostly lie: one axis inside the other, with and without gaps
        uint64_t size = t.dim;
        uint32_t order[3] = {0, 1, 2}, n[3] = {t.batch, t.length, t.heads};
        for (int i = 2; i > 0; --i) std::swap(order[i], order[pick(i + 1)]);
        for (uint32_t axis : order) {
            t.s[axis] = size + (pick(3) == 0 ? 8 * pick(5) : 0) - (pick(6) == 0 ? 8 : 0);
            size += t.s[axis] * (n[axis] - 1);
        }
    }
    return t;
}

static void self() {
    for (int n = 0; n < 20000; ++n) {
        const Layout t = random_layout();
        bool twice = false;
        elements(t, 0, &twice);
        okt_norm_rotary op = op_of(t.batch, t.length, t.heads, 0, t.dim);
        const uint64_t plain[3] = {(uint64_t)t.length * t.heads * t.dim, (uint64_t)t.heads * t.dim, t.dim};
        put(op.q_stride, plain);
        put(op.dq_stride, plain);
        put(op.q_out_stride, t.s);
        expect(okt_norm_rotary_forward(&op, at(1), nullptr, at(2), nullptr, nullptr), !twice, "self", t, 0);
        expect(okt_norm_rotary_backward(&op, nullptr, nullptr, at(1), nullptr, at(2), nullptr, nullptr, nullptr, nullptr, 0, nullptr), !twice, "self backward", t, 0);
    }
}

static void pairs() {
    for (int n = 0; n < 40000; ++n) {
        const Layout t = random_layout();
        bool twice = false;
        Layout k = t;
        k.heads = 1 + pick(4);
        const int64_t apart = pick(2) ? 8 * (int64_t)pick(200) - 800 : (int64_t)t.dim * (pick(60)) - 30 * (int64_t)t.dim;
        const std::set<int64_t> q_out = elements(t, 0, &twice), k_out = elements(k, apart, &twice);
        if (twice) continue;
        okt_norm_rotary op = op_of(t.batch, t.length, t.heads, k.heads, t.dim);
        for (uint64_t (*s)[3] : {&op.q_out_stride, &op.k_out_stride, &op.q_stride, &op.k_stride}) put(*s, t.s);
        char* far = at(2);
        expect(okt_norm_rotary_forward(&op, at(1), at(3), far, far + 2 * apart, nullptr), !meet(q_out, k_out), "outputs", t, apart);
        expect(okt_norm_rotary_forward(&op, at(1), far + 2 * apart, far, at(3), nullptr), !meet(q_out, k_out), "over the other's input", t, apart);
        const std::set<int64_t> q = elements(t, apart);
        expect(okt_norm_rotary_forward(&op, far + 2 * apart, at(1), far, at(3), nullptr), apart == 0 || !meet(q_out, q), "over its own input", t, apart);
    }
}

static void far() {
    const uint32_t most = (1u << 24) - 1;
    const uint64_t top = 1ull << 40;
    const struct { uint32_t batch, length, heads; uint64_t s[3]; int accepted; } t[] = {
        {1, most, 1, {0, 8, 0}, 1}, {1, most, 1, {0, 7, 0}, 0}, {4095, 4096, 16, {4096 * 128, 128, 8}, 1}, {4095, 4096, 16, {4096 * 128 - 8, 128, 8}, 0},
        {1, 1, 1u << 16, {0, 0, 8}, 1}, {2, 2, 2, {1u << 30, 1u << 20, 1u << 10}, 1},
        // an extent that no memory has
        {2, most / 2, 1, {top, top, 0}, 0}, {most, 1, 1, {top, 0, 0}, 0}, {4096, 4095, 1, {top, top - 8, 0}, 0},
        // lengths that would take long to look through one by one: either answer, as long as it comes
        {4096, 4095, 1u << 12, {8 * 4099, 8 * 4097, 8 * 4093}, -1}, {4096, 4095, 1u << 16, {8 * 65537, 8 * 65539, 8 * 65521}, -1}};
    for (const auto& x : t) {
        okt_norm_rotary op = op_of(x.batch, x.length, x.heads, 0, 8);
        put(op.q_out_stride, x.s);
        const auto begin = std::chrono::steady_clock::now();
        const int status = okt_norm_rotary_forward(&op, at(1), nullptr, at(2), nullptr, nullptr);
        const double seconds = std::chrono::duration<double>(std::chrono::steady_clock::now() - begin).count();
        expect(status, x.accepted < 0 ? status == OKT_OK : x.accepted, "far", {x.batch, x.length, x.heads, 8, {x.s[0], x.s[1], x.s[2]}}, 0);
        if (seconds > 0.05 && ++bad) std::printf("far: %u x %u x %u took %.2f s\n", x.batch, x.length, x.heads, seconds);
    }
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    if (what == "self") self();
    if (what == "pairs") pairs();
    if (what == "far") far();
    std::printf("%ld cases, %ld to refuse, %ld violations\n", cases, refused, bad);
    return bad || !cases ? 1 : 0;
}
