// Host check of what the layer's operators launch, without a GPU: this program stands in for the runtime's
// launch, which counts, looks at the sizes and does nothing.  Pointers are made up and never read.
//   sizes     every launch of a call that is accepted counts its work-items in 32 bits, and the sizes at the
//             edge of what the header allows are accepted, those past it refused (attention, dropout)
//   norm      outputs in the place of inputs, side by side and one after the other are taken
//   failed    a call ends with the first launch that fails
// Prints the number of cases and of violations.
#include <cstdio>
#include <cstring>
#include <initializer_list>

#include "okt.h"

struct Dim { uint32_t x, y, z; };
static int g_launches = 0, g_fail_at = 0, g_error = 0;       // launch number g_fail_at fails
static bool g_too_many = false;

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
    if ((uint64_t)grid.x * block.x >> 32 || (uint64_t)grid.y * block.y >> 16 || grid.z != 1) g_too_many = true;
    return g_launches == g_fail_at ? 9 : 0;
}
int hipGetLastError(void) {
    const int e = g_error;
    g_error = 0;
    return e;
}
}

static long cases = 0, bad = 0;
static void* const FAKE = (void*)0x10000;
static void* at(uint64_t n) { return (void*)(0x10000 + (n << 48)); }        // apart, whatever the sizes

static void judge(int status, bool accepted, const char* what, uint64_t a, uint64_t b, uint64_t c, uint64_t d) {
    ++cases;
    const bool fine = (status == OKT_OK) == accepted && !g_too_many && (status == OKT_OK || g_launches == 0) &&
                      (accepted ? g_launches > 0 : status == OKT_ERR_INVALID_ARG);
    if (!fine) {
        ++bad;
        std::printf("%s %llu %llu %llu %llu: status %d, %d launches%s\n", what, (unsigned long long)a, (unsigned long long)b,
                    (unsigned long long)c, (unsigned long long)d, status, g_launches, g_too_many ? ", too many work-items" : "");
    }
    g_launches = 0;
    g_too_many = false;
}

static uint64_t up(uint64_t n, uint64_t by) { return (n + by - 1) / by; }

static okt_attention attention_of(uint64_t batch, uint64_t heads, uint64_t kv_heads, uint64_t q_len, uint64_t k_len, uint32_t dim) {
    okt_attention op;
    std::memset(&op, 0, sizeof op);
    op.batch = (uint32_t)batch;
    op.heads = (uint32_t)heads;
    op.kv_heads = (uint32_t)kv_heads;
    op.q_len = (uint32_t)q_len;
    op.k_len = (uint32_t)k_len;
    op.head_dim = dim;
    op.dtype = OKT_BF16;
    op.scale = 1.0f;
    uint64_t* strides[] = {op.q_stride, op.k_stride, op.v_stride, op.o_stride, op.do_stride, op.dq_stride, op.dk_stride, op.dv_stride};
    for (uint64_t* s : strides) {
        s[0] = 1ull << 38;
        s[1] = dim;
        s[2] = 1ull << 32;
    }
    return op;
}

static const size_t WS = (size_t)1 << 62;
static int forward(const okt_attention& op) { return okt_attention_forward(&op, at(1), at(2), at(3), at(4), (float*)FAKE, FAKE, WS, nullptr); }
static int backward(const okt_attention& op) {
    return okt_attention_backward(&op, at(1), at(2), at(3), at(4), (float*)FAKE, at(5), at(6), at(7), at(8), FAKE, WS, nullptr);
}

static void attention(uint64_t batch, uint64_t heads, uint64_t kv_heads, uint64_t q_len, uint64_t k_len, uint32_t dim) {
    const okt_attention op = attention_of(batch, heads, kv_heads, q_len, k_len, dim);
    const uint64_t queries = up(q_len, 128) * batch * heads, keys = up(k_len, dim > 64 ? 64 : 128) * batch * kv_heads, most = 1ull << 24;
    judge(forward(op), batch * heads <= 1u << 20 && queries < most, "attention forward", batch * heads, batch * kv_heads, q_len, k_len);
    judge(backward(op), batch * heads <= 1u << 20 && queries < most && keys < most, "attention backward", batch * heads, batch * kv_heads, q_len, k_len);
}

static void dropout(uint64_t n, int dtype) {
    judge(okt_dropout(FAKE, FAKE, n, dtype, 0.1, (const uint64_t*)FAKE, 0, nullptr), n < (1ull << 37) - 8191, "dropout", n, dtype, 0, 0);
}

static void attentions() {
    for (uint32_t dim : {8u, 64u, 72u, 128u}) {
        for (uint64_t planes : {1ull, 3ull, 250ull, 513ull, 1ull << 10, 1ull << 14, (1ull << 20) - 1, 1ull << 20, (1ull << 20) + 1})
            for (uint64_t length : {1ull, 63ull, 64ull, 65ull, 128ull, 129ull, 1900ull, 2040ull, 2041ull, 2048ull, 2049ull, 1ull << 17, (1ull << 17) + 1, 1ull << 24})
                for (uint64_t other : {1ull, 64ull, 1025ull, 2048ull, 2049ull, 1ull << 20, 1ull << 24}) {
                    attention(1, planes, planes, length, other, dim);
                    attention(planes, 4, 1, length, other, dim);
                }
    }
}

static okt_residual_norm norm_of(bool gate) {
    okt_residual_norm op;
    std::memset(&op, 0, sizeof op);
    op.rows = 2000;
    op.width = 768;
    op.dtype = OKT_BF16;
    op.eps = 1e-5f;
    op.residual_scale = 1.0f;
    op.d_pre_weight = (const float*)FAKE;
    op.d_gate = gate ? (const float*)FAKE : nullptr;
    return op;
}

static void norms() {
    const auto place = [](uint64_t n) { return (void*)(0x100000 * n); };
    void *const u = place(1), *const x = place(2), *const h = place(3), *const y = place(4), *const dx = place(5), *const du = place(6);
    for (uint64_t stride : {0, 2 * 768}) {
        okt_residual_norm op = norm_of(false);
        op.rows = 100;
        for (uint64_t* s : {&op.u_stride, &op.x_stride, &op.h_stride, &op.y_stride, &op.dh_stride, &op.dy_stride, &op.dx_stride, &op.du_stride}) *s = stride;
        const auto after = [&](void* p) { return (char*)p + (stride ? 768 * 2 : 100 * 768 * 2); };
        const auto forward = [&](void* h_out, void* y_out) {
            judge(okt_residual_norm_forward(&op, u, x, h_out, y_out, nullptr, nullptr), true, "norm forward", (uint64_t)h_out, (uint64_t)y_out, stride, 0);
        };
        const auto backward = [&](void* dx_out, void* du_out) {
            judge(okt_residual_norm_backward(&op, nullptr, h, (const float*)FAKE, u, y, dx_out, du_out, nullptr, nullptr, nullptr, nullptr, nullptr, FAKE,
                                             (size_t)1 << 40, nullptr), true, "norm backward", (uint64_t)dx_out, (uint64_t)du_out, stride, 0);
        };
        forward(x, u);
        forward(u, x);
        forward(x, y);
        forward(h, u);
        forward(h, after(h));
        forward(after(u), after(x));
        backward(u, y);
        backward(h, u);
        backward(y, h);
        backward(dx, after(dx));
        backward(after(du), du);
        backward(after(u), after(h));
    }
}

// A call of `launches` launches, each of which fails in turn.
template <typename Call>
static void failing(const char* what, int launches, Call call) {
    for (int n = 0; n <= launches; ++n) {
        g_fail_at = n;
        const int status = call(), wanted = n ? n : launches;
        ++cases;
        if (g_launches != wanted || (status == OKT_OK) != (n == 0) || (n && status != OKT_ERR_HIP)) {
            ++bad;
            std::printf("%s, launch %d of %d fails: status %d, %d launches\n", what, n, launches, status, g_launches);
        }
        g_launches = g_fail_at = 0;
    }
}

static void failures() {
    const okt_attention few = attention_of(1, 2, 2, 1, 100000, 64), plain = attention_of(8, 64, 64, 256, 256, 64), odd = attention_of(1, 4, 2, 300, 3000, 128);
    failing("attention forward", 1, [&] { return forward(plain); });
    failing("attention forward in parts", 2, [&] { return forward(few); });
    failing("attention backward", 2, [&] { return backward(plain); });
    failing("attention backward in parts", 3, [&] { return backward(odd); });
    for (bool gate : {false, true}) {
        const okt_residual_norm op = norm_of(gate);
        failing("norm forward", 1, [&] { return okt_residual_norm_forward(&op, at(1), at(2), at(3), at(4), (float*)FAKE, nullptr); });
        failing("norm backward", 2, [&] {
            return okt_residual_norm_backward(&op, at(1), at(2), (const float*)FAKE, at(3), at(4), at(5), at(6), nullptr, nullptr,
                                              gate ? (float*)FAKE : nullptr, (float*)FAKE, nullptr, FAKE, WS, nullptr);
        });
    }
}

int main(int, char** what) {
    if (!std::strcmp(what[1], "attention")) attentions();
    if (!std::strcmp(what[1], "norm")) norms();
    if (!std::strcmp(what[1], "failed")) failures();
    if (!std::strcmp(what[1], "dropout"))
        for (int dtype : {OKT_F32, OKT_BF16, OKT_F16}) {
            const uint64_t most = (1ull << 37) - 8192;
            for (uint64_t n : {(uint64_t)1, (uint64_t)8193, (uint64_t)1 << 32, (uint64_t)1 << 36, most, most + 1, most + 8192, (uint64_t)1 << 40, (uint64_t)1 << 43}) dropout(n, dtype);
        }
    std::printf("%ld cases, %ld violations\n", cases, bad);
    return bad != 0;
}
