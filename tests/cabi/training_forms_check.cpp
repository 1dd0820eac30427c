// Which kernels the operators at the ends of a training step launch for given sizes, without a GPU: prints each launch's kernel, in order.
// Pointers are made up and never read.
//   loss ROWS WIDTH VOCAB WIDE        backward, with a bias, dW in fp32 where WIDE is 1
//   rotary BATCH LENGTH HEADS KV_HEADS DIM DTYPE BACKWARD
//   adamw STATE N N ...               lengths of tensors
#include <cstdio>
#include <cstdlib>
#include <cstring>

#include "launch_stub.h"
#include "okt.h"

static char* at(uint64_t n) { return (char*)(n << 44); }
static const size_t WS = (size_t)1 << 43;

static int loss(const std::vector<uint64_t>& n) {
    okt_cross_entropy op;
    std::memset(&op, 0, sizeof op);
    op.rows = n[0];
    op.width = (uint32_t)n[1];
    op.vocab = (uint32_t)n[2];
    op.dtype = OKT_BF16;
    op.dweight_dtype = n[3] ? OKT_F32 : OKT_BF16;
    op.dloss_stride = 1;
    op.d_bias = (const float*)at(9);
    return okt_cross_entropy_backward(&op, at(1), at(2), (const int64_t*)at(3), (const float*)at(4), (const float*)at(5), at(6), at(7), (float*)at(8), at(10), WS, nullptr);
}

static int rotary(const std::vector<uint64_t>& n) {
    okt_norm_rotary op;
    std::memset(&op, 0, sizeof op);
    op.batch = (uint32_t)n[0];
    op.length = (uint32_t)n[1];
    op.heads = (uint32_t)n[2];
    op.kv_heads = (uint32_t)n[3];
    op.head_dim = (uint32_t)n[4];
    op.dtype = (int32_t)n[5];
    op.kind = OKT_NORM_RMS;
    op.axes = 1;
    uint64_t* strides[] = {op.q_stride, op.k_stride, op.q_out_stride, op.k_out_stride, op.dq_stride, op.dk_stride};
    for (uint64_t* s : strides) {
        s[2] = n[4];
        s[1] = (n[2] + n[3]) * n[4];
        s[0] = s[1] * n[1];
    }
    op.d_q_weight = op.d_k_weight = (const float*)at(9);
    if (!n[6]) return okt_norm_rotary_forward(&op, at(1), at(2), at(3), at(4), nullptr);
    return okt_norm_rotary_backward(&op, at(1), at(2), at(3), at(4), at(5), at(6), (float*)at(7), (float*)at(8), at(10), WS, nullptr);
}

static int adamw(const std::vector<uint64_t>& n) {
    std::vector<okt_adamw_tensor> t(n.size() - 1);
    for (size_t i = 0; i < t.size(); ++i) {
        std::memset(&t[i], 0, sizeof t[i]);
        t[i].n = n[i + 1];
        t[i].rate_scale = 1.0;
        t[i].d_param = at(1) + (i << 38);
        t[i].d_grad = at(2) + (i << 38);
        t[i].d_m = at(3) + (i << 38);
        t[i].d_v = at(4) + (i << 38);
        if (n[0]) {
            t[i].d_m_scale = (float*)(at(5) + (i << 38));
            t[i].d_v_scale = (float*)(at(6) + (i << 38));
        }
    }
    const size_t need = okt_adamw_plan_bytes(t.data(), (uint32_t)t.size());
    std::vector<uint64_t> plan(need / 8 + 1);
    okt_adamw op;
    std::memset(&op, 0, sizeof op);
    op.tensors = (uint32_t)t.size();
    op.state = (int32_t)n[0];
    op.d_step = (const int64_t*)at(7);
    if (const int status = okt_adamw_plan(t.data(), op.tensors, op.state, plan.data(), need, &op.chunks)) return status;
    return okt_adamw_step(&op, at(8), nullptr);
}

int main(int argc, char** argv) {
    const std::string what = argc > 1 ? argv[1] : "";
    std::vector<uint64_t> n;
    for (int i = 2; i < argc; ++i) n.push_back(std::strtoull(argv[i], nullptr, 10));
    int status = -100;
    if (what == "loss" && n.size() == 4) status = loss(n);
    if (what == "rotary" && n.size() == 7) status = rotary(n);
    if (what == "adamw" && n.size() > 1) status = adamw(n);
    for (const Launched& l : g_launched) std::printf("%s\n", l.kernel.c_str());
    return status == OKT_OK ? 0 : 1;
}
