"""The rules that pick the linear layer's forms, compiled for the host."""
import ctypes as C
import os
import random
import subprocess

import pytest

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
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + CSRC, str(d / "r.cpp"), "-o", str(d / "r.so")], check=True)
    lib = C.CDLL(str(d / "r.so"))
    lib.form.argtypes = [C.c_int64, C.c_int64, C.c_int64, C.c_int]
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
