"""The sizes of tests/test_gpu_training_sizes.py take the forms of the kernels that they are there for, on the CPU: a host program in the runtime's
place says what is launched."""
import os
import shutil
import subprocess

import pytest

import paper_2201_07598_amd as okt
import test_gpu_training_sizes as sizes
from test_operators_abi import ROOT


@pytest.fixture(scope="module")
def launched(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    cabi, package = os.path.join(ROOT, "tests", "cabi"), os.path.join(ROOT, "paper_2201_07598_amd")
    exe = tmp_path_factory.mktemp("forms") / "forms_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"), "-I", cabi,
                    os.path.join(cabi, "training_forms_check.cpp"), "-L", package, "-lokt", "-ldl",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-Wl,-rpath," + package, "-o", str(exe)], check=True)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    env = {**os.environ, "LD_LIBRARY_PATH": os.pathsep.join([os.path.join(rocm, "lib"), os.environ.get("LD_LIBRARY_PATH", "")])}

    def run(*args):
        out = subprocess.run([str(exe), *map(str, args)], capture_output=True, text=True, env=env, timeout=100)
        assert out.returncode == 0, (out.stdout[-3000:], out.stderr[-2000:])
        return out.stdout.split("\n")[:-1]
    return run


@pytest.mark.parametrize("n", range(len(sizes.LOSSES)))
def test_pieces_and_products(launched, n):
    c, pieces, products = sizes.LOSSES[n]
    kernels = launched("loss", c["rows"], c["width"], c["vocab"], int(c.get("wide_dw", False)))
    assert sum("cross_entropy_gradient_kernel" in k for k in kernels) == pieces
    made = [k for k in kernels if "cross_entropy_products_kernel" in k]
    assert len(made) >= pieces and all(products in k for k in made)
    if products == sizes.LARGE:
        assert c["width"] > 256 or c["rows"] > 100_000


@pytest.mark.parametrize("n", range(len(sizes.ROTATIONS)))
def test_rotations(launched, n):
    c = sizes.ROTATIONS[n]
    for backward in (0, 1):
        for batch, around in ((c["batch"], "ELb1E"), (1, "ELb0E")):
            first = launched("rotary", batch, c["length"], c["heads"], c["kv_heads"], c["dim"], {"f32": 0, "bf16": 1, "f16": 2}[c["kind"]], backward)[0]
            assert "norm_rotary_" in first and around in first, first


@pytest.mark.parametrize("n", range(len(sizes.STEPS)))
def test_steps(launched, n):
    eight, lengths = sizes.STEPS[n][0], sizes.STEPS[n][-1]
    assert "adamw_kernelILb%dELb1E" % eight in launched("adamw", eight, *lengths)[0]
    for length in lengths:
        if length:
            assert "adamw_kernelILb%dELb0E" % eight in launched("adamw", eight, length)[0]


@pytest.mark.parametrize("rows,width,vocab", [(8192, 4096, 128_000), (131_072, 1024, 128_000), (16_384, 1024, 30_522)])
def test_a_workspace_has_room_for_the_parts_of_large_tiles(rows, width, vocab):
    """A wave of a large tile leaves two numbers for 128 columns of a row, and one for 64 rows of a column; d of a piece is a GiB or 4096 columns, and the rest
    are vectors and sums of dh and dW."""
    pad = lambda n, by: -(-n // by) * by  # noqa: E731
    stats = 8 * rows * pad(vocab, 256) // 128
    dbias = 4 * rows // 64 * pad(vocab, 256)
    d = 2 * rows * max(4096, 2 ** 30 // (2 * rows))
    others = rows * (2 + 4) * pad(width, 64) + 20 * rows + 4 * 256 * 256 * 256 + 2 * 256 * (d // rows) + (1 << 20)
    assert okt.okt_cross_entropy_workspace_bytes(rows, width, vocab) <= max(stats, dbias + d) + others
