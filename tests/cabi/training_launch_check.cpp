// Host check of what the operators at the ends of a training step launch, without a GPU: this program stands in for the runtime's
// launch, which counts, looks at the sizes and does nothing.  Pointers are made up and never read.
//   sizes     every launch of a call that is accepted counts its work-items in 32 bits and has some, and the edges of what the
//             header allows are accepted, what is past them refused before anything is launched
//   places    outputs of the rotation in the place of inputs, side by side and over one another
//   failed    a call ends with the first launch that fails
// Prints the number of cases and of violations.
#include <cstdio>
#include <cstring>
#include <initializer_list>
#include <vector>

#include "okt.h"

struct Dim { uint32_t x, y, z; };
static int g_launches = 0, g_fail_at = 0, g_error = 0;       // launch number g_fail_at fails
static bool g_wrong = false;

extern "C" {
static struct { Dim grid, block; size_t shared; void* stream; } g_next;
unsigned __hipPushCallConfiguration(Dim grid, Dim block, size_t shared, void* stream) {
    g_next = {grid, block, shared, stream};
    return 0;
}
int __hipPopCallConfiguration(Dim* grid, Dim* block, size_t* shared, void** stream) {
    *grid = g_next.grid;
    *block = g_next.block;
    *shared = g_next.shared;
    *stream = g_next.stream;
    return 0;
}
int hipLaunchKernel(const void*, Dim grid, Dim block, void**, size_t, void*) {
    ++g_launches;
    if (g_launches == g_fail_at) g_error = 9;                 // an invalid configuration
    if ((uint64_t)grid.x * block.x >> 32 || (uint64_t)grid.y * block.y >> 16 || grid.z != 1 || grid.x == 0 || grid.y == 0 || block.x == 0 || block.x > 1024) g_wrong = true;
    return g_launches == g_fail_at ? 9 : 0;
}
int hipGetLastError(void) {
    const int e = g_error;
    g_error = 0;
    return e;
}
}

static long cases = 0, bad = 0;
static void* at(uint64_t n) { return (void*)(0x10000 + (n << 48)); }        // apart, whatever the sizes
static const size_t WS = (size_t)1 << 60;

static void judge(int status, bool accepted, int launches, const char* what, uint64_t a, uint64_t b, uint64_t c, uint64_t d) {
    ++cases;
    const bool fine = (status == OKT_OK) == accepted && !g_wrong && (status == OKT_OK || g_launches == 0) &&
                      (launches < 0 || g_launches == launches) && (accepted || status == OKT_ERR_INVALID_ARG);
    if (!fine) {
        ++bad;
        std::printf("%s %llu %llu %llu %llu: status %d, %d launches%s\n", what, (unsigned long long)a, (unsigned long long)b,
                    (unsigned long long)c, (unsigned long long)d, status, g_launches, g_wrong ? ", of a wrong size" : "");
    }
    g_launches = 0;
    g_wrong = false;
}

// ------------------------------------------------------------------ cross entropy

static okt_cross_entropy ce_of(uint64_t rows, uint32_t width, uint32_t vocab, bool bias) {
    okt_cross_entropy op;
    std::memset(&op, 0, sizeof op);
    op.rows = rows;
    op.width = width;
    op.vocab = vocab;
    op.dtype = op.dweight_dtype = OKT_BF16;
    op.dloss_stride = 1;
    op.d_bias = bias ? (const float*)at(9) : nullptr;
    return op;
}
static int ce_forward(const okt_cross_entropy& op) {
    return okt_cross_entropy_forward(&op, at(1), at(2), (const int64_t*)at(3), (float*)at(4), (float*)at(5), at(10), WS, nullptr);
}
static int ce_backward(const okt_cross_entropy& op, bool dh = true, bool dw = true) {
    return okt_cross_entropy_backward(&op, at(1), at(2), (const int64_t*)at(3), (const float*)at(4), (const float*)at(5), dh ? at(6) : nullptr,
                                      dw ? at(7) : nullptr, op.d_bias ? (float*)at(8) : nullptr, at(10), WS, nullptr);
}

static void cross_entropies() {
    const uint64_t top = 1u << 22;
    for (uint64_t rows : {1ull, 127ull, 128ull, 129ull, 2048ull, 2049ull, 16384ull, 1ull << 20, 1ull << 22})
        for (uint64_t vocab : {1ull, 255ull, 257ull, 10007ull, 128000ull, 1ull << 20, 1ull << 22})
            for (uint64_t width : {8ull, 64ull, 776ull, 4096ull, 1ull << 15}) {
                const okt_cross_entropy op = ce_of(rows, (uint32_t)width, (uint32_t)vocab, true);
                // rows are laid side by side first, but for a few of few tiles
                const bool few = rows <= 128 || (rows + 255) / 256 * ((vocab + 255) / 256) < 200;
                const int listed = rows > 2048 ? 2 : few ? 0 : 1;
                judge(ce_forward(op), true, listed + 2, "cross entropy forward", rows, vocab, width, 0);
                const size_t need = okt_cross_entropy_workspace_bytes(rows, (uint32_t)width, (uint32_t)vocab);
                judge(ce_backward(op), true, -1, "cross entropy backward", rows, vocab, width, 0);
                judge(need >= 2 * rows * width ? OKT_OK : OKT_ERR_HIP, true, 0, "workspace", rows, vocab, width, need);
            }
    judge(ce_forward(ce_of(top + 1, 64, 100, false)), false, 0, "rows", top + 1, 0, 0, 0);
    judge(ce_forward(ce_of(10, 64, (uint32_t)top + 1, false)), false, 0, "vocab", top + 1, 0, 0, 0);
    judge(ce_forward(ce_of(10, 64, 0, false)), false, 0, "vocab", 0, 0, 0, 0);
    for (uint32_t width : {0u, 4u, 12u, (1u << 15) + 8}) judge(ce_forward(ce_of(10, width, 100, false)), false, 0, "width", width, 0, 0, 0);
    judge(ce_forward(ce_of(0, 64, 100, false)), true, 0, "no rows", 0, 0, 0, 0);
    judge(ce_backward(ce_of(0, 64, 100, true)), true, -1, "no rows backward", 0, 0, 0, 0);
    // one product for the logits, one for each gradient that is wanted, and the sums
    judge(ce_backward(ce_of(300, 64, 100, false), true, false), true, 4, "dh alone", 0, 0, 0, 0);
    judge(ce_backward(ce_of(300, 64, 100, false), false, true), true, 3, "dweight alone", 0, 0, 0, 0);
}

// ------------------------------------------------------------------ rotation

static okt_norm_rotary rotary_of(uint32_t batch, uint32_t length, uint32_t heads, uint32_t kv_heads, uint32_t dim, bool norm) {
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
    op.d_q_weight = op.d_k_weight = norm ? (const float*)at(9) : nullptr;
    uint64_t* strides[] = {op.q_stride, op.k_stride, op.q_out_stride, op.k_out_stride, op.dq_stride, op.dk_stride};
    for (uint64_t* s : strides) {
        const uint64_t row = (uint64_t)(heads + 2 * kv_heads) * dim;
        s[0] = row * (length ? length : 1);
        s[1] = row;
        s[2] = dim;
    }
    return op;
}

static void rotations() {
    for (uint32_t dim : {8u, 64u, 72u, 128u, 136u, 256u})
        for (uint32_t heads : {1u, 3u, 16u, 40u, 1u << 12, 1u << 16})
            for (uint64_t tokens : {1ull, 2ull, 1000ull, 1ull << 20, (1ull << 24) - 1})
                for (bool norm : {false, true}) {
                    if (tokens * heads * dim >> 42) continue;            // made-up tensors would meet
                    const okt_norm_rotary op = rotary_of((uint32_t)(tokens > 7 ? tokens / 7 : 1), tokens > 7 ? 7 : (uint32_t)tokens, heads, 1, dim, norm);
                    judge(okt_norm_rotary_forward(&op, at(1), at(2), at(3), at(4), nullptr), true, 1, "rotation forward", dim, heads, tokens, norm);
                    float* w = norm ? (float*)at(7) : nullptr;
                    const int status = okt_norm_rotary_backward(&op, at(1), at(2), at(3), at(4), at(5), at(6), w, nullptr, at(8), WS, nullptr);
                    judge(status, true, norm ? 2 : 1, "rotation backward", dim, heads, tokens, norm);
                }
    for (const okt_norm_rotary& op : {rotary_of(1u << 12, 1u << 12, 1, 1, 64, true), rotary_of(1, 1, (1u << 16) + 1, 1, 64, true), rotary_of(1, 1, 0, 0, 64, true),
                                      rotary_of(1, 1, 1, 1, 12, true), rotary_of(1, 1, 1, 1, 264, true)})
        judge(okt_norm_rotary_forward(&op, at(1), at(2), at(3), at(4), nullptr), false, 0, "rotation refused", op.batch, op.length, op.heads, op.head_dim);
}

// Parts of one projection: elements from the buffer's first to each tensor's.
static void rotation_places() {
    const uint32_t H = 6, G = 2, D = 64, S = 5, B = 3;
    const int64_t row = (H + 2 * G) * D;
    okt_norm_rotary op = rotary_of(B, S, H, G, D, true);
    char* base = (char*)at(1);
    const auto run = [&](int64_t q, int64_t k, int64_t qo, int64_t ko) { return okt_norm_rotary_forward(&op, base + 2 * q, base + 2 * k, base + 2 * qo, base + 2 * ko, nullptr); };
    const int64_t far = 1 << 20, k0 = H * D;
    judge(run(0, k0, 0, k0), true, 1, "in place", 0, 0, 0, 0);
    judge(run(2 * G * D, 0, 2 * G * D, 0), true, 1, "in place, keys first", 0, 0, 0, 0);
    judge(run(0, k0, far, far + k0), true, 1, "elsewhere", 0, 0, 0, 0);
    judge(run(0, k0, far, far + k0 - 8), false, 0, "outputs overlap", 0, 0, 0, 0);
    for (int64_t by : {(int64_t)8, (int64_t)D, row, (int64_t)row * S, row * S - row, -row, row + 2 * (int64_t)D})
        judge(run(0, k0, by, far + k0), false, 0, "over the queries", (uint64_t)by, 0, 0, 0);
    judge(run(0, k0, k0, far), false, 0, "queries over the keys", 0, 0, 0, 0);
    judge(run(0, k0, far, (H - G) * D), false, 0, "keys over the last queries", 0, 0, 0, 0);
    judge(run(0, k0, far, (H + G) * D), true, 1, "keys over the values", 0, 0, 0, 0);
    judge(run(0, k0, row * S * B, far), true, 1, "behind", 0, 0, 0, 0);
    // a weight and the positions right before and behind the queries' output, and one element further in
    const int64_t size = ((B * S - 1) * row + H * D) * 2;
    char* out = base + 2 * far;
    op.position_stride[0] = S;
    op.position_stride[1] = 1;
    for (int in : {0, 4}) {
        op.d_q_weight = (const float*)(out - 4 * D + in);
        judge(run(0, k0, far, 2 * far), in == 0, in == 0, "behind a weight", in, 0, 0, 0);
        op.d_q_weight = (const float*)(out + size - in);
        judge(run(0, k0, far, 2 * far), in == 0, in == 0, "before a weight", in, 0, 0, 0);
        op.d_q_weight = nullptr;
        op.d_positions = (const int32_t*)(out - 4 * B * S + in);
        judge(run(0, k0, far, 2 * far), in == 0, in == 0, "behind the positions", in, 0, 0, 0);
        op.d_positions = nullptr;
    }
    // heads with q, k, v of each side by side
    for (uint64_t* s : {op.q_stride, op.k_stride, op.q_out_stride, op.k_out_stride}) s[2] = 3 * D;
    op.heads = op.kv_heads = 3;
    judge(run(0, D, 0, D), true, 1, "each head's, in place", 0, 0, 0, 0);
    judge(run(0, D, 2 * D, far), true, 1, "each head's, over its values", 0, 0, 0, 0);
    judge(run(0, D, D, far), false, 0, "each head's, over its keys", 0, 0, 0, 0);
    op.k_out_stride[2] = 0;
    judge(run(0, D, far, 2 * far), false, 0, "keys all in one place", 0, 0, 0, 0);
}

// ------------------------------------------------------------------ AdamW

static void steps() {
    std::vector<okt_adamw_tensor> t(300);
    for (size_t i = 0; i < t.size(); ++i) {
        std::memset(&t[i], 0, sizeof t[i]);
        char* base = (char*)at(1) + (i << 38);
        t[i].n = i % 7 == 0 ? 0 : i * i + 1;
        t[i].d_param = base;
        t[i].d_grad = (char*)at(2) + 64;                     // shared
        t[i].d_m = base + (1ull << 36);
        t[i].d_v = base + (2ull << 36);
        t[i].rate_scale = 1.0;
    }
    t[299].n = 1ull << 34;
    const size_t need = okt_adamw_plan_bytes(t.data(), 300);
    std::vector<uint64_t> plan(need / 8 + 1);
    uint32_t chunks = 0;
    judge(okt_adamw_plan(t.data(), 300, OKT_STATE_F32, plan.data(), need, &chunks), true, 0, "plan", need, 0, 0, 0);
    uint64_t want = 0;
    for (const auto& x : t) want += (x.n + 4095) / 4096;
    judge(chunks == want ? OKT_OK : OKT_ERR_HIP, true, 0, "chunks", chunks, want, 0, 0);
    okt_adamw op;
    std::memset(&op, 0, sizeof op);
    op.tensors = 300;
    op.chunks = chunks;
    op.beta1 = 0.9;
    op.beta2 = 0.999;
    op.d_step = (const int64_t*)at(3);
    judge(okt_adamw_step(&op, at(4), nullptr), true, 1, "step", chunks, 0, 0, 0);
    op.chunks = 0;
    judge(okt_adamw_step(&op, at(4), nullptr), true, 0, "a step of nothing", 0, 0, 0, 0);
    op.chunks = (1u << 24) - 1;
    judge(okt_adamw_step(&op, at(4), nullptr), true, 1, "the longest step", op.chunks, 0, 0, 0);
    op.chunks = 1u << 24;
    judge(okt_adamw_step(&op, at(4), nullptr), false, 0, "a longer step", op.chunks, 0, 0, 0);
    t[5].n = 1ull << 36;
    judge(okt_adamw_plan_bytes(t.data(), 300) == 0 ? OKT_ERR_INVALID_ARG : OKT_OK, false, 0, "too long", 0, 0, 0, 0);
}

// ------------------------------------------------------------------ failures

template <typename F>
static void fails(const char* what, const F& call) {
    g_launches = 0;
    call();
    const int all = g_launches;
    for (int n = 1; n <= all; ++n) {
        g_launches = 0;
        g_fail_at = n;
        const int status = call();
        ++cases;
        if (status != OKT_ERR_HIP || g_launches != n) {
            ++bad;
            std::printf("%s: launch %d of %d failed: status %d after %d launches\n", what, n, all, status, g_launches);
        }
    }
    g_fail_at = g_launches = g_error = 0;
    g_wrong = false;
}

static void failures() {
    for (uint64_t rows : {100ull, 5000ull})
        for (uint32_t vocab : {100u, 300000u}) {
            const okt_cross_entropy op = ce_of(rows, 64, vocab, true);
            fails("cross entropy forward", [&] { return ce_forward(op); });
            fails("cross entropy backward", [&] { return ce_backward(op); });
        }
    const okt_norm_rotary op = rotary_of(2, 10, 4, 2, 64, true);
    fails("rotation forward", [&] { return okt_norm_rotary_forward(&op, at(1), at(2), at(3), at(4), nullptr); });
    fails("rotation backward", [&] { return okt_norm_rotary_backward(&op, at(1), at(2), at(3), at(4), at(5), at(6), (float*)at(7), nullptr, at(8), WS, nullptr); });
    okt_adamw step;
    std::memset(&step, 0, sizeof step);
    step.tensors = step.chunks = 1;
    step.d_step = (const int64_t*)at(3);
    fails("step", [&] { return okt_adamw_step(&step, at(4), nullptr); });
}

int main(int argc, char** argv) {
    const char* what = argc > 1 ? argv[1] : "";
    if (!std::strcmp(what, "sizes")) {
        cross_entropies();
        rotations();
        steps();
    } else if (!std::strcmp(what, "places")) {
        rotation_places();
    } else if (!std::strcmp(what, "failed")) {
        failures();
    }
    std::printf("%ld cases, %ld violations\n", cases, bad);
    return bad || !cases ? 1 : 0;
}
