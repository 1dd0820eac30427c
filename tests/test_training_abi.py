"""The operators at the ends of a training step at the C ABI, on the CPU: the structs the binding packs are those the header
declares, arguments out of range are refused on the host, the binding names what is wrong with a tensor, the index arithmetic of the
matrix products covers everything once, and launches have the sizes they can have."""
import ctypes
import os
import shutil
import subprocess

import pytest
import torch

import paper_2201_07598_amd as okt
from paper_2201_07598_amd import binding
from test_operators_abi import FAKE, INVALID, OK, ROOT, WORKSPACE, offsets_in_c, offsets_packed

AT = [FAKE << n for n in range(14)]            # aligned, apart, never dereferenced


def test_packed_structs_match_the_header(tmp_path):
    entropy = ["rows", "width", "vocab", "dtype", "dweight_dtype", "dloss_stride", "reserved", "d_bias", "h_stride", "weight_stride",
               "dh_stride", "dweight_stride"]
    assert offsets_in_c(tmp_path, "okt_cross_entropy", entropy) == offsets_packed(binding._CROSS_ENTROPY.format)
    tensor = ["d_param", "d_grad", "d_m", "d_v", "d_copy", "d_m_scale", "d_v_scale", "n", "weight_decay", "rate_scale", "param_dtype",
              "grad_dtype", "copy_dtype", "reserved"]
    assert offsets_in_c(tmp_path, "okt_adamw_tensor", tensor) == offsets_packed(binding._ADAMW_TENSOR.format)
    step = ["tensors", "chunks", "state", "site", "lr", "beta1", "beta2", "eps", "d_step", "d_lr", "d_grad_scale", "d_skip", "d_seed"]
    assert offsets_in_c(tmp_path, "okt_adamw", step) == offsets_packed(binding._ADAMW.format)
    rotary = ["batch", "length", "heads", "kv_heads", "head_dim", "rot_dim", "dtype", "kind", "eps", "adjacent", "axes", "reserved"]
    rest = ["d_inv_freq", "d_positions", "position_stride[0]", "position_stride[1]", "d_q_weight", "d_k_weight"]
    rest += [f"{t}_stride[{i}]" for t in ("q", "k", "q_out", "k_out", "dq", "dk") for i in range(3)]
    names = rotary + [f"axis_of_pair[{i}]" for i in range(128)] + rest
    assert offsets_in_c(tmp_path, "okt_norm_rotary", names) == offsets_packed(binding._ROTARY.format)


# ------------------------------------------------------------------ cross entropy

ENTROPY = dict(rows=4, width=64, vocab=100, dtype=1, dw=1, step=1, bias=0)


def entropy_struct(**change):
    a = {**ENTROPY, **change}
    return binding._CROSS_ENTROPY.pack(a["rows"], a["width"], a["vocab"], a["dtype"], a["dw"], a["step"], 0, a["bias"], 0, 0, 0, 0)


def test_cross_entropy_refusals():
    lib = okt.load_library()
    B = AT[11]

    def forward(h=AT[0], w=AT[1], y=AT[2], loss=AT[3], lse=AT[4], ws=AT[9], ws_bytes=1 << 40, **change):
        return lib.okt_cross_entropy_forward(entropy_struct(**change), h, w, y, loss, lse, ws, ws_bytes, None)

    def backward(h=AT[0], w=AT[1], y=AT[2], lse=AT[3], g=AT[4], dh=AT[5], dw_out=AT[6], db=None, ws=AT[9], ws_bytes=1 << 40, **change):
        return lib.okt_cross_entropy_backward(entropy_struct(**change), h, w, y, lse, g, dh, dw_out, db, ws, ws_bytes, None)

    shared = [{"rows": (1 << 22) + 1}, {"width": 0}, {"width": 12}, {"width": (1 << 15) + 8}, {"vocab": 0}, {"vocab": (1 << 22) + 1}, {"dtype": 0},
              {"dtype": 3}, {"step": 2}, {"bias": B + 2}, {"w": None}, {"h": None}, {"y": None}]
    for bad in shared:
        assert forward(**bad) == INVALID, bad
        assert backward(**bad) == INVALID, bad
    for strides in ((56, 0, 0, 0), (68, 0, 0, 0), (0, 56, 0, 0), (0, (1 << 20) + 8, 0, 0), (0, 0, 56, 0), (0, 0, 0, 56), (0, 0, 0, (1 << 20) + 8)):
        op = binding._CROSS_ENTROPY.pack(4, 64, 100, 1, 1, 1, 0, 0, *strides)
        assert lib.okt_cross_entropy_backward(op, *AT[:7], None, AT[9], 1 << 40, None) == INVALID, strides
        assert lib.okt_cross_entropy_forward(op, *AT[:5], AT[9], 1 << 40, None) == INVALID, strides
    for bad in ({"loss": None}, {"h": AT[0] + 8}, {"w": AT[1] + 2}, {"y": AT[2] + 4}, {"loss": AT[3] + 2}, {"lse": AT[4] + 1}, {"lse": AT[3]}, {"loss": AT[0]},
                {"loss": AT[1] + 4}, {"lse": AT[2] + 8}):
        assert forward(**bad) == INVALID, bad
    assert forward(bias=B, lse=B + 396) == INVALID
    for bad in ({"dw": 2}, {"dw": 3}, {"lse": None}, {"g": None}, {"dh": AT[5] + 8}, {"dw_out": AT[6] + 8}, {"db": AT[7]}, {"dh": None, "dw_out": None},
                {"dh": AT[0]}, {"dh": AT[0] + 128}, {"dw_out": AT[1]}, {"dh": AT[6] + 64}, {"dw_out": AT[4] - 64}, {"bias": B, "db": B},
                {"bias": B, "db": AT[7] + 2}, {"dw": 0, "dw_out": AT[6] + 2}, {"dw": 0, "dw_out": AT[5] - 8}):
        assert backward(**bad) == INVALID, bad
    for bad in ({"ws": None}, {"ws": AT[9] + 16}, {"ws_bytes": 4096}):
        assert forward(**bad) == WORKSPACE, bad
        assert backward(**bad) == WORKSPACE, bad
    assert forward(rows=0, h=None, y=None, loss=None) == OK
    assert okt.okt_cross_entropy_workspace_bytes(4, 12, 100) == 0 and okt.okt_cross_entropy_workspace_bytes(0, 64, 100) > 0


# ------------------------------------------------------------------ rotation

ROTARY = dict(batch=2, length=8, heads=4, kv_heads=2, dim=64, rot=64, dtype=1, kind=1, eps=1e-6, adjacent=0, axes=1, table=b"", freq=AT[10],
              positions=0, by=(0, 0), q_weight=0, k_weight=0, strides=(4096, 512, 64) * 6)


def rotary_struct(**change):
    a = {**ROTARY, **change}
    return binding._ROTARY.pack(a["batch"], a["length"], a["heads"], a["kv_heads"], a["dim"], a["rot"], a["dtype"], a["kind"], a["eps"],
                                a["adjacent"], a["axes"], 0, a["table"], a["freq"], a["positions"], *a["by"], a["q_weight"], a["k_weight"], *a["strides"])


def test_rotary_refusals():
    lib = okt.load_library()

    def forward(q=AT[0], k=AT[1], qo=AT[2], ko=AT[3], **change):
        return lib.okt_norm_rotary_forward(rotary_struct(**change), q, k, qo, ko, None)

    def backward(q=AT[0], k=AT[1], dq=AT[2], dk=AT[3], qo=AT[4], ko=AT[5], qw=None, kw=None, ws=AT[9], ws_bytes=1 << 30, **change):
        return lib.okt_norm_rotary_backward(rotary_struct(**change), q, k, dq, dk, qo, ko, qw, kw, ws, ws_bytes, None)

    def strides(place, value):
        s = [4096, 512, 64] * 6
        s[place] = value
        return {"strides": tuple(s)}

    W = AT[11]
    shared = [{"batch": 1 << 12, "length": 1 << 12}, {"heads": 0, "kv_heads": 0}, {"heads": (1 << 16) + 1}, {"dim": 0}, {"dim": 60}, {"dim": 264}, {"rot": 72},
              {"rot": 4}, {"dtype": 3}, {"kind": 2}, {"eps": -1.0}, {"eps": float("nan")}, {"eps": float("inf")}, {"axes": 0}, {"axes": 9}, {"axes": 2},
              {"table": b"\0\1"}, {"freq": 0}, {"freq": AT[10] + 2}, {"positions": FAKE + 2}, {"q_weight": W + 2}, {"k_weight": W + 1},
              {"qo": None}, {"ko": None}, {"qo": AT[4] + 1}, strides(6, 56), strides(7, 8), strides(8, 32), strides(11, 0), strides(0, 1 << 41), strides(8, 1 << 31)]
    for bad in shared:
        assert forward(**bad) == INVALID, bad
        assert backward(**bad) == INVALID, bad
    for bad in ({"q": None}, {"k": None}, {"q": AT[0] + 1}, {"qo": AT[1]}, {"qo": AT[3]}, {"ko": AT[0] + 128}):
        assert forward(**bad) == INVALID, bad
    for bad in ({"dq": None}, {"dk": None}, {"qw": AT[7]}, {"kw": AT[7]}, {"q_weight": W, "q": None}, {"k_weight": W, "k": None},
                {"q_weight": W, "qw": AT[7] + 2}, {"qo": AT[3]}, {"ko": AT[2]}, {"qo": AT[5]}, {"k_weight": W, "qo": AT[1]}, {"heads": 0, "q_weight": W, "qw": AT[7]}):
        assert backward(**bad) == INVALID, bad
    for bad in ({"ws": None}, {"ws": AT[9] + 16}, {"ws_bytes": 64}):
        assert backward(q_weight=W, qw=AT[7], **bad) == WORKSPACE, bad
    assert forward(batch=0) == OK and backward(length=0) == OK
    assert okt.okt_norm_rotary_workspace_bytes(1, 1, 1, 0, 12) == 0 and okt.okt_norm_rotary_workspace_bytes(0, 1, 1, 0, 64) == 256
    assert okt.okt_norm_rotary_workspace_bytes(8, 4096, 16, 4, 128) == 1024 * 2 * 128 * 4


def test_rotary_weights_gradients_are_apart():
    struct = rotary_struct(q_weight=AT[11], k_weight=AT[11])
    for to in (AT[7], AT[7] + 4 * 63):
        args = (struct, *AT[:6], AT[7], to, AT[9], 1 << 30, None)
        assert okt.load_library().okt_norm_rotary_backward(*args) == INVALID


def test_rotary_outputs_are_apart_from_parameters():
    """An output over a weight, the frequencies or the positions, from their first to their last element, and a weight's gradient over anything."""
    lib, last = okt.load_library(), (4096 + 7 * 512 + 3 * 64 + 63) * 2          # of the queries
    parts = [({"q_weight": AT[11]}, 256), ({"k_weight": AT[11]}, 256), ({"freq": AT[11]}, 128), ({"positions": AT[11], "by": (8, 1)}, 64)]
    for change, size in parts:
        struct = rotary_struct(**change)
        for to in (AT[11], AT[11] + size - 2, AT[11] - last):
            assert lib.okt_norm_rotary_forward(struct, AT[0], AT[1], to, AT[3], None) == INVALID, change
            assert lib.okt_norm_rotary_backward(struct, *AT[:4], to, AT[5], None, None, None, 0, None) == INVALID, change
    struct = rotary_struct(q_weight=AT[11], k_weight=AT[12], positions=AT[13])
    for to in (AT[0] + last - 2, AT[1], AT[2], AT[3] - 252, AT[4], AT[5] + 128, AT[10] + 124, AT[11], AT[12] + 252, AT[13]):
        assert lib.okt_norm_rotary_backward(struct, *AT[:6], to, None, AT[9], 1 << 30, None) == INVALID, to
        assert lib.okt_norm_rotary_backward(struct, *AT[:6], None, to, AT[9], 1 << 30, None) == INVALID, to


@pytest.mark.timeout(30)
def test_rotary_without_a_batch_takes_any_length():
    lib = okt.load_library()
    for sizes in ({"batch": 0, "length": (1 << 32) - 1}, {"batch": (1 << 32) - 1, "length": 0}):
        assert lib.okt_norm_rotary_forward(rotary_struct(**sizes), *AT[:4], None) == OK
        assert okt.okt_norm_rotary_workspace_bytes(sizes["batch"], sizes["length"], 8, 8, 64) == 256


# ------------------------------------------------------------------ AdamW

TENSOR = dict(p=AT[0], g=AT[1], m=AT[2], v=AT[3], copy=0, ms=0, vs=0, n=1000, decay=0.0, rate=1.0, pt=0, gt=0, ct=1)


def tensor_struct(**change):
    a = {**TENSOR, **change}
    return binding._ADAMW_TENSOR.pack(a["p"], a["g"], a["m"], a["v"], a["copy"], a["ms"], a["vs"], a["n"], a["decay"], a["rate"], a["pt"], a["gt"], a["ct"], 0)


def plan_of(*tensors, state=0, room=0, count=None, buffer=None):
    lib, table = okt.load_library(), b"".join(tensors)
    count = len(tensors) if count is None else count
    need = lib.okt_adamw_plan_bytes(table, count)
    host, chunks = ctypes.create_string_buffer(need + 64), ctypes.c_uint32(77)
    at = (ctypes.addressof(host) + 15) // 16 * 16 if buffer is None else buffer
    status = lib.okt_adamw_plan(table, count, state, at, need + room, ctypes.cast(ctypes.pointer(chunks), ctypes.c_void_p))
    return status, chunks.value, need


def test_plan_refusals():
    one = tensor_struct()
    assert plan_of(one) == (OK, 1, 256)
    assert plan_of(tensor_struct(n=4097))[1] == 2 and plan_of(tensor_struct(n=0, p=0, g=0, m=0, v=0))[:2] == (OK, 0)
    assert okt.okt_adamw_plan_bytes([4097, 0, 1]) == 512 and okt.okt_adamw_plan_bytes([1 << 36]) == 0
    for bad in ({"p": 0}, {"g": 0}, {"m": 0}, {"v": 0}, {"p": AT[0] + 2}, {"g": AT[1] + 1}, {"m": AT[2] + 2}, {"pt": 3}, {"gt": -1},
                {"copy": AT[4], "ct": 0}, {"copy": AT[4] + 1}, {"ms": AT[4]}, {"ms": AT[4], "vs": AT[5]}, {"decay": -0.1}, {"decay": float("nan")},
                {"rate": -1.0}, {"rate": float("inf")},
                {"m": AT[0]}, {"v": AT[0] + 3996}, {"g": AT[0] + 4}, {"copy": AT[0] + 2}, {"m": AT[3] - 4}):
        assert plan_of(tensor_struct(**bad))[0] == INVALID, bad
    eight = dict(ms=AT[4], vs=AT[5])
    assert plan_of(tensor_struct(**eight), state=1)[0] == OK
    for bad in ({}, {"ms": AT[4]}, {"ms": AT[4], "vs": AT[4]}, {"ms": AT[4], "vs": AT[4] + 12}, {"ms": AT[4], "vs": AT[3] + 996}, {"ms": AT[4] + 2, "vs": AT[5]}):
        assert plan_of(tensor_struct(**bad), state=1)[0] == INVALID, bad
    assert plan_of(tensor_struct(ms=AT[4], vs=AT[4] + 16), state=1)[0] == OK              # four blocks each
    # the same tensor twice, a shared gradient, neighbours
    assert plan_of(one, one)[0] == INVALID
    far = dict(p=AT[6], m=AT[7], v=AT[8])
    assert plan_of(one, tensor_struct(**far))[0] == OK
    assert plan_of(one, tensor_struct(**{**far, "p": AT[0] + 4000}))[0] == OK
    assert plan_of(one, tensor_struct(**{**far, "p": AT[0] + 3996}))[0] == INVALID
    assert plan_of(one, tensor_struct(**{**far, "p": AT[1]}))[0] == INVALID                # over another's gradient
    assert plan_of(one, state=2)[0] == INVALID and plan_of(one, count=0)[0] == INVALID
    assert plan_of(one, room=-1)[0] == WORKSPACE and plan_of(one, buffer=0)[0] == WORKSPACE


def test_step_refusals():
    lib = okt.load_library()

    def step(plan=AT[0], tensors=1, chunks=1, state=0, lr=0.1, b1=0.9, b2=0.999, eps=1e-8, t=AT[1], d_lr=0, scale=0, skip=0, seed=0):
        return lib.okt_adamw_step(binding._ADAMW.pack(tensors, chunks, state, 0, lr, b1, b2, eps, t, d_lr, scale, skip, seed), plan, None)

    for bad in ({"plan": None}, {"plan": AT[0] + 8}, {"tensors": 0}, {"chunks": 1 << 24}, {"state": 2}, {"lr": float("nan")}, {"lr": float("inf")}, {"b1": 1.0},
                {"b1": -0.1}, {"b2": 1.0}, {"b2": float("nan")}, {"eps": -1.0}, {"eps": float("inf")}, {"t": 0}, {"t": AT[1] + 4}, {"d_lr": AT[2] + 2},
                {"scale": AT[2] + 1}, {"skip": AT[2] + 3}, {"seed": AT[2] + 4}):
        assert step(**bad) == INVALID, bad
    assert step(chunks=0) == OK


# ------------------------------------------------------------------ the binding

def test_binding_names_what_is_wrong():
    h, w = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(10, 64, dtype=torch.bfloat16)
    y, f = torch.zeros(4, dtype=torch.int64), torch.zeros(4)
    with pytest.raises(TypeError, match="bfloat16 or float16"):
        okt.okt_cross_entropy_forward(h.float(), w.float(), y, f, f, None)
    with pytest.raises(ValueError, match="agree in width"):
        okt.okt_cross_entropy_forward(h, w[:, :32], y, f, f, None)
    with pytest.raises(ValueError, match="rows, width"):
        okt.okt_cross_entropy_forward(h[0], w, y, f, f, None)
    with pytest.raises(TypeError, match="CUDA"):
        okt.okt_cross_entropy_forward(h, w, y, f, f, None)
    q, freq = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16), torch.zeros(32)
    with pytest.raises(ValueError, match="batch, length, heads"):
        okt.okt_norm_rotary_forward(q[0], None, q[0], None, freq)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        okt.okt_norm_rotary_forward(q.double(), None, q, None, freq)
    with pytest.raises(TypeError, match="CUDA"):
        okt.okt_norm_rotary_forward(q, None, q, None, freq)
    p = torch.zeros(10)
    e = torch.zeros(10, dtype=torch.float8_e4m3fn)
    for error, match, args, options in (
            (ValueError, "empty", ([], [], [], []), {}), (ValueError, "one tensor a parameter", ([p], [p, p], [p], [p]), {}),
            (TypeError, "grads is required", ([p], None, [p], [p]), {}), (TypeError, "float8_e4m3fn", ([p], [p], [p.half()], [p]), {}),
            (TypeError, "belong to", ([p], [p], [e], [e]), {}), (TypeError, "belong to", ([p], [p], [p], [p]), {"m_scales": [p], "v_scales": [p]}),
            (TypeError, "CUDA", ([p], [p], [p], [p]), {}), (ValueError, "one value a tensor", ([p], [p], [p], [p]), {"weight_decay": [0.1, 0.2]})):
        with pytest.raises(error, match=match):
            okt.okt_adamw_plan(*args, **options)


# ------------------------------------------------------------------ host programs

def test_product_layout_covers_everything_once(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "layout_check"
    subprocess.run([gxx, "-O2", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2201_07598_amd", "csrc"),
                    os.path.join(ROOT, "tests", "cabi", "product_layout_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and " 0 violations" in out.stdout, out.stdout


@pytest.mark.parametrize("what", ["sizes", "places", "failed"])
def test_launches(tmp_path, what):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    package, exe = os.path.join(ROOT, "paper_2201_07598_amd"), tmp_path / "launch_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "cabi", "training_launch_check.cpp"), "-L", package, "-lokt",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-Wl,-rpath," + package, "-o", str(exe)], check=True)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    env = {**os.environ, "LD_LIBRARY_PATH": os.pathsep.join([os.path.join(rocm, "lib"), os.environ.get("LD_LIBRARY_PATH", "")])}
    out = subprocess.run([str(exe), what], capture_output=True, text=True, env=env, timeout=100)
    assert out.returncode == 0 and " 0 violations" in out.stdout, (out.stdout[-3000:], out.stderr[-2000:])
