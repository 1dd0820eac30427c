"""The layer's operators at the C ABI, on the CPU: the structs the binding packs are those the
header declares, arguments out of range are refused on the host, the binding names what is
wrong with a tensor, and the index arithmetic of the kernels covers everything once."""
import ctypes
import os
import shutil
import struct
import subprocess

import pytest
import torch

import paper_2201_07598_amd as okt
from paper_2201_07598_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
OK, INVALID, WORKSPACE = 0, -1, -2
FAKE = 0x10000                 # aligned, never dereferenced on these paths


def offsets_in_c(tmp_path, name, members):
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no gcc")
    src, exe = tmp_path / "offsets.c", tmp_path / "offsets"
    lines = "".join(f'    printf("%zu ", offsetof({name}, {m}));\n' for m in members)
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "okt.h"\nint main(void) {\n'
                   f'{lines}    printf("%zu\\n", sizeof({name}));\n    return 0;\n}}\n')
    subprocess.run([gcc, "-std=c99", "-I", os.path.join(ROOT, "include"), str(src), "-o", str(exe)], check=True)
    return [int(n) for n in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]


def offsets_packed(fmt):
    """Offsets of the members of a packed format, repeats of one letter counted one by one."""
    out, at, count = [], 0, ""
    for ch in fmt[1:]:
        if ch.isdigit():
            count += ch
            continue
        for _ in range(int(count or 1)):
            out.append(at)
            at += struct.calcsize("=" + ch)
        count = ""
    return out + [at]


def test_packed_structs_match_the_header(tmp_path):
    norm = ["rows", "width", "dtype", "kind", "eps", "residual_scale", "site", "dropout_p", "d_seed",
            "d_post_weight", "d_post_bias", "d_gate", "rows_per_gate", "d_pre_weight", "d_pre_bias", "u_stride",
            "x_stride", "h_stride", "y_stride", "dh_stride", "dy_stride", "dx_stride", "du_stride"]
    assert offsets_in_c(tmp_path, "okt_residual_norm", norm) == offsets_packed(binding._NORM.format)
    attention = ["batch", "heads", "kv_heads", "q_len", "k_len", "head_dim", "dtype", "causal", "scale", "site",
                 "dropout_p", "d_seed", "d_q_lens", "d_k_lens"]
    attention += [f"{t}_stride[{i}]" for t in ("q", "k", "v", "o", "do", "dq", "dk", "dv") for i in range(3)]
    assert offsets_in_c(tmp_path, "okt_attention", attention) == offsets_packed(binding._ATTENTION.format)


def dropout(x=FAKE, y=FAKE, n=64, dtype=1, p=0.1, seed=FAKE):
    return okt.load_library().okt_dropout(x, y, n, dtype, p, seed, 0, None)


def test_dropout_refusals():
    assert dropout(n=0, x=None, y=None) == OK
    for bad in ({"x": None}, {"y": None}, {"seed": None}, {"x": FAKE + 8}, {"y": FAKE + 2}, {"seed": FAKE + 4},
                {"dtype": 3}, {"dtype": -1}, {"p": -0.01}, {"p": 1.01}, {"p": float("nan")}, {"n": (1 << 43) + 1}):
        assert dropout(**bad) == INVALID, bad


NORM = dict(rows=4, width=64, dtype=1, kind=0, eps=1e-5, scale=1.0, site=0, p=0.0, seed=0, post_w=0, post_b=0, gate=0,
            share=0, pre_w=FAKE, pre_b=FAKE, strides=(0,) * 8)


def norm_struct(**change):
    a = {**NORM, **change}
    return binding._NORM.pack(a["rows"], a["width"], a["dtype"], a["kind"], a["eps"], a["scale"], a["site"], a["p"],
                              a["seed"], a["post_w"], a["post_b"], a["gate"], a["share"], a["pre_w"], a["pre_b"], *a["strides"])


def test_norm_refusals():
    lib = okt.load_library()

    def forward(u=FAKE, x=FAKE, h=FAKE, y=FAKE, stats=FAKE, **change):
        return lib.okt_residual_norm_forward(norm_struct(**change), u, x, h, y, stats, None)

    def backward(u=FAKE, h=FAKE, stats=FAKE, dh=FAKE, dy=FAKE, dx=FAKE, du=FAKE, pw=None, pb=None, g=None, w=None, b=None,
                 ws=FAKE, ws_bytes=1 << 24, **change):
        return lib.okt_residual_norm_backward(norm_struct(**change), u, h, stats, dh, dy, dx, du, pw, pb, g, w, b, ws, ws_bytes, None)

    shared = [{"width": 7}, {"width": 8193}, {"rows": (1 << 40) + 1}, {"dtype": 3}, {"kind": 2}, {"eps": -1.0},
              {"eps": float("nan")}, {"scale": float("nan")}, {"p": 1.5}, {"p": 0.5}, {"p": 0.5, "seed": FAKE + 4},
              {"post_b": FAKE}, {"pre_w": 0}, {"pre_w": FAKE + 4}, {"strides": (63, 0, 0, 0, 0, 0, 0, 0)},
              {"strides": (0, 0, 0, 0, 0, 0, 0, (1 << 20) + 1)}]
    for bad in shared:
        assert forward(**bad) == INVALID, bad
        assert backward(**bad) == INVALID, bad
    for bad in ({"u": None}, {"x": None}, {"y": None}, {"h": FAKE + 1}, {"stats": FAKE + 8},
                {"pre_w": 0, "pre_b": 0, "y": FAKE}, {"pre_w": 0, "pre_b": 0, "y": None, "h": None}):
        assert forward(**bad) == INVALID, bad
    for bad in ({"h": None}, {"dy": None}, {"stats": None}, {"dx": None}, {"du": None}, {"pw": FAKE}, {"g": FAKE},
                {"b": FAKE, "pre_b": 0}, {"post_w": FAKE, "u": None}, {"gate": FAKE, "u": None},
                {"pre_w": 0, "pre_b": 0}, {"w": FAKE + 2}):
        assert backward(**bad) == INVALID, bad
    other = FAKE + 4096                                             # in an input's place, with another stride
    assert forward(u=other, strides=(0, 72, 0, 0, 0, 0, 0, 0), y=other + 4096) == INVALID
    assert backward(u=None, h=other, dy=other + 4096, du=other + 8192, strides=(0, 0, 0, 0, 72, 0, 0, 0)) == INVALID
    assert forward(rows=0, u=None, x=None) == OK
    for bad in ({"ws": None}, {"ws": FAKE + 16}, {"ws_bytes": 255}):
        assert backward(**bad) == WORKSPACE, bad
    # 512 workgroups of 196 rows each would be 100,352 rows: 511 are enough, and each leaves five sums
    assert okt.okt_residual_norm_workspace_bytes(100_000, 1024, 0) == 5 * 511 * 1024 * 4
    assert okt.okt_residual_norm_workspace_bytes(4, 7, 0) == 0 and okt.okt_residual_norm_workspace_bytes(0, 64, 0) > 0


ATTENTION = dict(batch=2, heads=4, kv_heads=2, q_len=8, k_len=8, dim=64, dtype=1, causal=0, scale=0.125, site=0, p=0.0,
                 seed=0, q_lens=0, k_lens=0, strides=(2048, 256, 64) * 8)


def attention_struct(**change):
    a = {**ATTENTION, **change}
    return binding._ATTENTION.pack(a["batch"], a["heads"], a["kv_heads"], a["q_len"], a["k_len"], a["dim"], a["dtype"],
                                   a["causal"], a["scale"], a["site"], a["p"], a["seed"], a["q_lens"], a["k_lens"], *a["strides"])


def test_attention_refusals():
    lib = okt.load_library()

    def forward(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, ws=FAKE, ws_bytes=1 << 30, **change):
        return lib.okt_attention_forward(attention_struct(**change), q, k, v, o, lse, ws, ws_bytes, None)

    def backward(q=FAKE, k=FAKE, v=FAKE, o=FAKE, lse=FAKE, do=FAKE, dq=FAKE, dk=FAKE, dv=FAKE, ws=FAKE, ws_bytes=1 << 30, **change):
        return lib.okt_attention_backward(attention_struct(**change), q, k, v, o, lse, do, dq, dk, dv, ws, ws_bytes, None)

    shared = [{"kv_heads": 0}, {"heads": 0}, {"heads": 5}, {"dim": 0}, {"dim": 12}, {"dim": 136}, {"dtype": 0}, {"dtype": 3},
              {"scale": 0.0}, {"scale": -1.0}, {"scale": float("nan")}, {"scale": float("inf")}, {"p": 0.5}, {"p": -0.5},
              {"q_len": (1 << 24) + 1}, {"batch": 1 << 20}, {"q_lens": FAKE + 2}, {"strides": (2048, 252, 64) * 8},
              {"strides": (2048, 1 << 25, 64) * 8}, {"strides": (2048, 0, 64) * 8}, {"q": FAKE + 8}, {"k": None}, {"v": None}, {"o": None}, {"q": None}]
    for bad in shared:
        assert forward(**bad) == INVALID, bad
        assert backward(**bad) == INVALID, bad
    for bad in ({"lse": None}, {"do": None}, {"dq": None}, {"dk": None}, {"dv": FAKE + 8}):
        assert backward(**bad) == INVALID, bad
    for bad in ({"ws": None}, {"ws": FAKE + 16}, {"ws_bytes": 64}):
        assert backward(**bad) == WORKSPACE, bad
    # few rows, many keys: the forward pass needs room for its parts as well
    long = {"q_len": 1, "k_len": 100_000, "heads": 2, "kv_heads": 1, "batch": 1}
    assert forward(ws=None, ws_bytes=0, **long) == WORKSPACE
    assert forward(q_len=0) == OK and forward(batch=0) == OK and backward(batch=0) == OK


def test_attention_workspace():
    need = okt.okt_attention_workspace_bytes(2, 16, 4, 4096, 4096, 128)
    assert need % 256 == 0 and need >= 2 * 16 * 4096 * 8
    for shape in ((1, 1, 1, 1, 1, 8), (1, 12, 12, 1, 4096, 64), (32, 16, 16, 512, 512, 64), (1, 4, 1, 4096, 3, 128)):
        assert okt.okt_attention_workspace_bytes(*shape) >= 256
    # sizes beyond 32 bits do not wrap
    assert okt.okt_attention_workspace_bytes(1024, 128, 128, 1 << 20, 1, 128) >= 1024 * 128 * (1 << 20) * 8


def test_binding_names_what_is_wrong():
    x = torch.zeros(4, 64)
    with pytest.raises(TypeError, match="CUDA"):
        okt.okt_dropout(x, x, 0.1, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError, match="seed"):
        okt.okt_dropout(x, x, 0.1, None)
    with pytest.raises(ValueError, match="length"):
        okt.okt_dropout(x, x[:1], 0.1, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        okt.okt_residual_norm_forward(x.double(), x, x, x, None, pre_weight=x[0])
    with pytest.raises(ValueError, match="rows, width"):
        okt.okt_residual_norm_forward(x[0], x, x, x, None, pre_weight=x[0])
    with pytest.raises(TypeError, match="CUDA"):
        okt.okt_residual_norm_backward(x, x, x, x, x, x, x, x, pre_weight=x[0])
    q = torch.zeros(1, 2, 2, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="batch, length, heads"):
        okt.okt_attention_forward(q[0], q, q, q, None)
    with pytest.raises(ValueError, match="agree"):
        okt.okt_attention_forward(q, q[..., :32], q, q, None)
    with pytest.raises(TypeError, match="CUDA"):
        okt.okt_attention_forward(q, q, q, q, None)


def test_attention_layout_covers_everything_once(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    exe = tmp_path / "layout_check"
    subprocess.run([gxx, "-O2", "-std=c++17", "-Wall", "-Werror", "-I",
                    os.path.join(ROOT, "paper_2201_07598_amd", "csrc"),
                    os.path.join(ROOT, "tests", "cabi", "attention_layout_check.cpp"), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True)
    assert out.returncode == 0 and " 0 violations" in out.stdout, out.stdout


def launch_check(tmp_path, *args):
    """The host program that stands in for the runtime's launch, linked with the library."""
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    package, exe = os.path.join(ROOT, "paper_2201_07598_amd"), tmp_path / "launch_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"),
                    os.path.join(ROOT, "tests", "cabi", "launch_check.cpp"), "-L", package, "-lokt",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-Wl,-rpath," + package, "-o", str(exe)], check=True)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    env = {**os.environ, "LD_LIBRARY_PATH": os.pathsep.join([os.path.join(rocm, "lib"), os.environ.get("LD_LIBRARY_PATH", "")])}
    out = subprocess.run([str(exe), *args], capture_output=True, text=True, env=env, timeout=100)
    assert out.returncode == 0 and " 0 violations" in out.stdout, (out.stdout[-3000:], out.stderr[-2000:])


def test_attention_launches_within_the_sizes_of_a_launch(tmp_path):
    launch_check(tmp_path, "attention")


def test_dropout_launches_within_the_sizes_of_a_launch(tmp_path):
    launch_check(tmp_path, "dropout")


def test_a_call_ends_with_the_first_launch_that_fails(tmp_path):
    launch_check(tmp_path, "failed")


def test_assembly_names_the_registers_it_sets():
    """A statement that sets m0 says so; otherwise the compiler may keep something of its own there."""
    import glob
    import re
    setting = 0
    for path in sorted(glob.glob(os.path.join(ROOT, "paper_2201_07598_amd", "csrc", "*"))):
        for statement in re.findall(r"\basm\b[^;]*?\(.*?\)\s*;", open(path).read(), flags=re.S):
            if re.search(r"s_\w+ m0\b", statement):
                setting += 1
                assert '"m0"' in statement.rsplit(":", 1)[1], (path, statement)
    assert setting


def test_norm_refuses_outputs_that_overlap():
    """Outputs over each other, and over inputs at another place than row by row; halves of one buffer are apart."""
    lib = okt.load_library()
    U, X, H, Y = (FAKE << n for n in range(1, 5))
    two, apart = (128,) * 8, 64 * 2                                        # rows of 64 in two bytes each, beside another tensor's

    def forward(u=U, x=X, h=H, y=Y, **change):
        return lib.okt_residual_norm_forward(norm_struct(**change), u, x, h, y, None, None)

    def backward(h=H, dh=U, dy=Y, dx=X, du=FAKE << 5, **change):
        return lib.okt_residual_norm_backward(norm_struct(**change), None, h, FAKE << 6, dh, dy, dx, du, None, None, None, None, None,
                                              FAKE << 7, 1 << 24, None)

    for bad in ({"y": H}, {"y": H + 2}, {"y": H + 3 * 128}, {"h": X, "y": X}, {"h": X + 2}, {"y": U - 2}, {"h": U + 128},
                {"y": H + apart - 2, "strides": two}, {"y": H + 126, "strides": two}, {"rows": 1, "y": H + 126}, {"rows": 1, "h": X + 2}):
        assert forward(**bad) == INVALID, bad
    for bad in ({"du": X}, {"du": X - 126}, {"du": X + 3 * 128}, {"dx": H + 2}, {"du": Y + 128}, {"dx": U - 2},
                {"du": X + 130, "strides": (128,) * 8, "dx": X + 4}, {"rows": 1, "du": X + 2}):
        assert backward(**bad) == INVALID, bad


def test_norm_takes_outputs_in_the_place_of_inputs_and_side_by_side(tmp_path):
    launch_check(tmp_path, "norm")


def test_attention_refuses_outputs_that_overlap():
    lib = okt.load_library()
    at = {n: FAKE << i for i, n in enumerate(("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv", "ws"))}

    def forward(ws_bytes=1 << 30, change=None, **place):
        a = {**at, **place}
        return lib.okt_attention_forward(attention_struct(**(change or {})), a["q"], a["k"], a["v"], a["o"], a["lse"], a["ws"], ws_bytes, None)

    def backward(ws_bytes=1 << 30, change=None, **place):
        a = {**at, **place}
        return lib.okt_attention_backward(attention_struct(**(change or {})), *(a[n] for n in ("q", "k", "v", "o", "lse", "do", "dq", "dk", "dv", "ws")), ws_bytes, None)

    for name in ("q", "k", "v"):
        assert forward(o=at[name]) == INVALID, name
        assert forward(o=at[name] + 112) == INVALID, name
    for out in ("dq", "dk", "dv"):
        for name in ("q", "k", "v", "o", "do", *({"dq", "dk", "dv"} - {out})):
            assert backward(**{out: at[name]}) == INVALID, (out, name)


def test_attention_refuses_outputs_whose_places_are_the_same_memory():
    """One vector for all sequences, or for all heads: inputs may be broadcast so, outputs not."""
    lib, at = okt.load_library(), [FAKE << i for i in range(10)]
    strides = [2048, 256, 64] * 8
    for tensor in (3, 5, 6, 7):
        for axis in (0, 2):
            for step in (0, 56):
                same = list(strides)
                same[3 * tensor + axis] = step
                op = attention_struct(strides=same)
                if tensor == 3:
                    assert lib.okt_attention_forward(op, *at[:6], 1 << 30, None) == INVALID, (axis, step)
                else:
                    assert lib.okt_attention_backward(op, *at, 1 << 30, None) == INVALID, (tensor, axis, step)


def test_dropout_refuses_an_output_that_overlaps_its_input():
    for dtype, size in ((0, 4), (1, 2)):
        for y in (FAKE + 16, FAKE - 16, FAKE + 64 * size - 16, FAKE - 64 * size + 16):
            assert dropout(y=y, dtype=dtype) == INVALID, (dtype, y)
