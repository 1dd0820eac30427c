"""Which places the rotation may write, on the CPU: every call is looked at by a host program that lists the elements one by one, with
the launches taken by a stand-in for the runtime."""
import os
import shutil
import subprocess

import pytest

import paper_2201_07598_amd as okt
from test_operators_abi import INVALID, ROOT
from test_training_abi import AT, rotary_struct


@pytest.fixture(scope="module")
def places(tmp_path_factory):
    gxx = shutil.which("g++")
    if gxx is None:
        pytest.skip("no g++")
    cabi, package = os.path.join(ROOT, "tests", "cabi"), os.path.join(ROOT, "paper_2201_07598_amd")
    exe = tmp_path_factory.mktemp("places") / "places_check"
    subprocess.run([gxx, "-O1", "-std=c++17", "-Wall", "-Werror", "-rdynamic", "-I", os.path.join(ROOT, "include"), "-I", cabi,
                    os.path.join(cabi, "rotary_places_check.cpp"), "-L", package, "-lokt", "-ldl",
                    "-Wl,--unresolved-symbols=ignore-in-shared-libs", "-Wl,-rpath," + package, "-o", str(exe)], check=True)
    rocm = os.environ.get("ROCM_PATH", "/opt/rocm")
    env = {**os.environ, "LD_LIBRARY_PATH": os.pathsep.join([os.path.join(rocm, "lib"), os.environ.get("LD_LIBRARY_PATH", "")])}

    def run(what):
        out = subprocess.run([str(exe), what], capture_output=True, text=True, env=env, timeout=100)
        assert out.returncode == 0 and " 0 violations" in out.stdout, (out.stdout[-3000:], out.stderr[-2000:])
    return run


def forward(q, k, q_out, k_out, **change):
    return okt.load_library().okt_norm_rotary_forward(rotary_struct(**change), q, k, q_out, k_out, None)


def test_tensors_of_like_strides(places):
    places("pairs")


def test_keys_between_the_steps_of_queries():
    """Heads 128 apart, tokens 192: token 1's first key is token 0's third query, though no axis alone leads there."""
    change = dict(batch=1, length=2, heads=3, kv_heads=3, strides=(10_000, 192, 128) * 6)
    for apart in (64, 128, 192, 256, 320):
        assert forward(AT[0], AT[1], AT[2], AT[2] + 2 * apart, **change) == INVALID, apart


def test_an_output_that_overlaps_itself(places):
    places("self")


def test_ends_of_sizes_and_strides(places):
    places("far")


@pytest.mark.parametrize("sizes,strides", [
    ((1, 2, 2), (10_000, 64, 64)), ((2, 2, 1), (512, 512, 64)), ((2, 1, 2), (64, 512, 64)), ((3, 3, 4), (8 * 64, 4 * 64 - 8, 64)), ((1, 3, 3), (0, 96, 192))])
def test_two_heads_in_one_place(sizes, strides):
    """Strides that are all a head's length or more, and yet two heads share elements."""
    batch, length, heads = sizes
    apart = (1 << 16, 1 << 12, 1 << 8)
    change = dict(batch=batch, length=length, heads=heads, kv_heads=1)
    assert forward(*AT[:4], strides=apart * 2 + strides + apart * 3, **change) == INVALID
    struct = rotary_struct(strides=apart * 2 + strides + apart * 3, **change)
    assert okt.load_library().okt_norm_rotary_backward(struct, None, None, *AT[2:6], None, None, None, 0, None) == INVALID
