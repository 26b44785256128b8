"""The rules that pick the linear layer's forms, compiled for the host."""
import ctypes as C
import os
import random
import subprocess

import pytest

from paper_1912_02057_amd import binding as B
from test_linear import SIZES
from test_linear_forms import BACKWARD, FORWARD

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_02057_amd", "csrc")


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("rules")
    (d / "r.cpp").write_text("""#include "choice.h"
extern "C" int form(int64_t M, int64_t N, int64_t K, int z) { return (int)rtn::linear_form(M, N, K, z != 0); }
extern "C" void wgrad(int64_t M, int64_t N, int64_t K, int* out)
{
    const rtn::WgradForm f = rtn::wgrad_form(M, N, K);
    out[0] = f.tile, out[1] = f.splits;
}
extern "C" int64_t run(int64_t M, int64_t N) { return rtn::grad_blocks_per_run(M, N); }
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = C.CDLL(str(d / "r.so"))
    lib.form.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int]
    lib.run.argtypes, lib.run.restype = [C.c_int64, C.c_int64], C.c_int64
    lib.wgrad.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.POINTER(C.c_int)]

    def wgrad(M, N, K):
        out = (C.c_int * 2)()
        lib.wgrad(M, N, K, out)
        return tuple(out)
    lib.wgrad_form = wgrad
    return lib


def test_no_run_of_the_weight_gradient_is_empty(rules):
    """Every block of a split product has tokens: the last run begins before the end."""
    rng = random.Random(1)
    sizes = [(1216, 64, 64), (2112, 64, 64), (0, 64, 64), (1, 1, 1), (64 * 19, 300, 200)]
    sizes += [(int(2 ** rng.uniform(0, 17)), int(2 ** rng.uniform(0, 14)), int(2 ** rng.uniform(0, 14))) for _ in range(4000)]
    sizes.append(((1 << 31) - 2048, 1 << 21, 1 << 21))
    for M, N, K in sizes:
        tile, splits = rules.wgrad_form(M, N, K)
        steps = (M + 63) // 64
        assert tile in (64, 128, 256) and 1 <= splits <= 16
        assert splits == 1 or (splits - 1) * -(-steps // splits) < steps, (M, N, K, tile, splits)


def test_sizes_reach_every_form_of_the_product(rules):
    """Tiles over more steps than their ring has stages and with all waves at work, and every form whose rows may be copied first both ways."""
    few, split32, split32x64, split64, tile128, tile256 = range(6)
    seen = set()
    for M, N, K, start in FORWARD:
        f, ld = rules.form(M, N, K, 0), K + start
        assert f == rules.form(M, N, K, 1)                   # with a checkpoint
        copied = B.lib().rtn_linear_workspace_bytes(C.c_void_p(0x10000 + 2 * start), ld, M, N, K, 0) > 0
        if f in (tile128, tile256):
            assert N >= 256 and K > 4 * 64
        seen.add((f, copied))
    assert {(tile128, False), (tile128, True), (tile256, False), (tile256, True), (split64, False), (split64, True),
            (split32, True), (split32x64, True)} <= seen, seen


def test_sizes_reach_every_form_of_the_gradients(rules):
    """Each tile of the weight gradient alone and split, few steps and many, edges inside a tile, and each length of a run of dz's sums."""
    seen, steps = set(), set()
    for M, N, K in BACKWARD + SIZES:
        tile, splits = rules.wgrad_form(M, N, K)
        seen.add((tile, splits > 1))
        if splits == 1:
            steps.add((tile, min((M + 63) // 64, 5)))
    assert seen == {(t, s) for t in (64, 128, 256) for s in (False, True)}
    assert {(64, n) for n in (1, 2, 3, 5)} | {(128, n) for n in (1, 2, 3, 4)} | {(256, 5)} <= steps
    assert all(any(rules.wgrad_form(M, N, K)[0] == t and M % 64 and N % t and K % t for M, N, K in BACKWARD) for t in (64, 128, 256))
    assert {rules.run(M, N) for M, N, K in BACKWARD} == {1, 2, 8}
