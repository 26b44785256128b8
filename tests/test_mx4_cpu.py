"""What the entry points of the microscaled 4-bit operators and of the norms refuse, on a host without a GPU: every check comes before
any launch."""
import ctypes as C
import os
import subprocess

import numpy as np
import pytest

from paper_1912_02057_amd import binding as B
from test_linear_cpu import BIG, FAKE, HALF, L, ODD, OTHER, _refuses  # noqa: F401 (L is a fixture)

N, S, U, A, W = B.RTN_ERR_NULL, B.RTN_ERR_SHAPE, B.RTN_ERR_UNSUPPORTED, B.RTN_ERR_ALIGN, B.RTN_ERR_WORKSPACE
FOUR = C.c_void_p(0x10004)
MOST = 1 << 21


def _empty(call, ok, zero, none):
    """A call with no rows is one with nothing to do, its matrices may be NULL."""
    assert call(*[0 if i == zero else None if i in none else v for i, v in enumerate(ok)]) == B.RTN_OK


def test_sizes(L):  # noqa: F811
    assert L.rtn_mx4_bytes(1, 1) == 1024 + 256
    assert L.rtn_mx4_bytes(17, 129) == 2 * 2 * 1024 + 2 * 256
    assert L.rtn_mx4_bytes(65, 128) == 5 * 1024 + 2 * 256
    assert L.rtn_mx4_bytes(4096, 4096) == 4096 * 4096 * 17 // 32
    assert L.rtn_mx4_bytes(0, 5) == 0 and L.rtn_mx4_bytes(5, 0) == 0 and L.rtn_mx4_bytes(-1, 5) == 0
    assert L.rtn_mx4_bytes(MOST, MOST) == MOST * MOST * 17 // 32 and L.rtn_mx4_bytes(MOST + 1, 5) == 0 == L.rtn_mx4_bytes(5, MOST + 1)
    assert L.rtn_mx4_linear_workspace_bytes(100, 64, 200) == L.rtn_mx4_bytes(100, 200)
    assert L.rtn_mx4_linear_workspace_bytes(0, 64, 200) == 0 == L.rtn_mx4_linear_workspace_bytes(100, 0, 200)
    assert L.rtn_mx4_linear_backward_workspace_bytes(100, 64, 0) == 0 == L.rtn_mx4_linear_backward_workspace_bytes(0, 64, 64)
    assert L.rtn_mx4_linear_backward_workspace_bytes(100, 64, 64) >= L.rtn_mx4_bytes(100, 64) + L.rtn_mx4_bytes(64, 100) + 64 * 4
    assert L.rtn_norm_backward_workspace_bytes(0, 64, 1) == 0 == L.rtn_norm_backward_workspace_bytes(5, 64, 0)
    assert L.rtn_norm_backward_workspace_bytes(5, 16385, 5) == 0
    assert L.rtn_norm_backward_workspace_bytes(5, 64, 5) == L.rtn_norm_backward_workspace_bytes(5, 64, 1 << 40) >= 4 * 6 * 64 * 4


def test_pack_refuses(L):  # noqa: F811
    #     0 dt       1 x  2 ldx 3 R 4 C 5 p   6 pb 7 pt   8 ptb 9 seed 10 stream
    ok = [B.RTN_BF16, FAKE, 64, 100, 64, FAKE, BIG, OTHER, BIG, FAKE, None]
    _refuses(L.rtn_mx4_pack, ok, [
        ({1: None}, N), ({5: None, 7: None}, N), ({0: 3}, U), ({0: -1}, U), ({2: 63}, S), ({2: 1 << 32}, S), ({3: -1}, S), ({4: 0}, S),
        ({3: MOST + 1}, S), ({4: MOST + 1, 2: 1 << 22}, S), ({1: ODD}, A), ({0: B.RTN_F32, 1: HALF}, A), ({5: HALF}, A), ({7: FOUR}, A),
        ({9: FOUR}, A), ({6: 7 * 1024 + 2 * 256 - 1}, W), ({8: 4 * 1024 + 255}, W)])
    _empty(L.rtn_mx4_pack, ok, 3, (1,))


def test_unpack_refuses(L):  # noqa: F811
    ok = [B.RTN_F16, FAKE, BIG, 100, 64, OTHER, 64, None]
    _refuses(L.rtn_mx4_unpack, ok, [({1: None}, N), ({5: None}, N), ({0: 3}, U), ({3: -1}, S), ({4: 0}, S), ({6: 63}, S), ({5: ODD}, A),
                                    ({0: B.RTN_F32, 5: HALF}, A), ({1: HALF}, A), ({2: 7 * 1024 + 511}, W)])
    _empty(L.rtn_mx4_unpack, ok, 3, (1, 5))


def test_linear_refuses(L):  # noqa: F811
    #     0 dt       1 x  2 ldx 3 xp 4 xpb 5 w  6 wb 7 M 8 N 9 K 10 b  11 act 12 r 13 ldr 14 y 15 ldy 16 z 17 ldz 18 ws 19 wsb 20 stream
    ok = [B.RTN_BF16, FAKE, 64, None, 0, FAKE, BIG, 100, 64, 64, FAKE, 0, FAKE, 64, OTHER, 64, FAKE, 64, FAKE, BIG, None]
    _refuses(L.rtn_mx4_linear, ok, [
        ({1: None}, N), ({5: None}, N), ({14: None}, N), ({0: B.RTN_F32}, U), ({0: 7}, U), ({11: 4}, U), ({11: -1}, U), ({7: -1}, S), ({8: 0}, S),
        ({9: 0}, S), ({2: 63}, S), ({13: 63}, S), ({15: 63}, S), ({17: 63}, S), ({15: 1 << 32}, S), ({7: MOST + 1}, S),
        ({1: ODD}, A), ({10: ODD}, A), ({12: ODD}, A), ({14: ODD}, A), ({16: ODD}, A), ({5: HALF}, A), ({3: HALF, 4: BIG}, A), ({18: HALF}, A),
        ({6: 4 * 1024 + 255}, W), ({3: FAKE, 4: 7 * 1024 + 511}, W), ({18: None}, W), ({19: 7 * 1024 + 511}, W)])
    _empty(L.rtn_mx4_linear, ok, 7, (1, 14))


def test_backward_refuses(L):  # noqa: F811
    #     0 dt       1 dy 2 ld 3 z 4 ldz 5 act 6 wt 7 wb 8 xt 9 xb 10 M 11 N 12 K 13 seed 14 dx 15 lddx 16 dw 17 type 18 db 19 ws 20 wsb 21 st
    ok = [B.RTN_F16, FAKE, 64, FAKE, 64, B.RTN_ACT_RELU, FAKE, BIG, FAKE, BIG, 100, 64, 96, FAKE, OTHER, 96, OTHER, B.RTN_F32, OTHER, FAKE, BIG, None]
    _refuses(L.rtn_mx4_linear_backward, ok, [
        ({14: None, 16: None, 18: None}, N), ({1: None}, N), ({3: None}, N), ({6: None}, N), ({8: None}, N), ({0: B.RTN_F32}, U), ({5: 4}, U),
        ({17: B.RTN_BF16}, U), ({2: 63}, S), ({4: 63}, S), ({15: 95}, S), ({10: -1}, S), ({11: 0}, S), ({12: 0}, S), ({10: MOST + 1}, S),
        ({1: ODD}, A), ({3: ODD}, A), ({14: ODD}, A), ({16: HALF}, A), ({18: ODD}, A), ({6: HALF}, A), ({8: HALF}, A), ({13: FOUR}, A), ({19: HALF}, A),
        ({7: 6 * 1024 + 511}, W), ({9: 6 * 1024 + 511}, W), ({19: None}, W), ({20: 4000}, W)])


def test_norm_refuses(L):  # noqa: F811
    f = C.c_float
    #     0 dt       1 kind 2 x 3 ldx 4 M 5 C 6 w  7 b   8 eps 9 u 10 ldu 11 stream
    ok = [B.RTN_BF16, 0, FAKE, 64, 100, 64, FAKE, FAKE, f(1e-6), OTHER, 64, None]
    _refuses(L.rtn_norm, ok, [({2: None}, N), ({6: None}, N), ({9: None}, N), ({0: 2}, U), ({1: 2}, U), ({1: -1}, U), ({4: -1}, S), ({5: 0}, S),
                              ({5: 16385, 3: 20000, 10: 20000}, S), ({3: 63}, S), ({10: 63}, S), ({8: f(-1)}, S), ({8: f(np.nan)}, S), ({2: ODD}, A),
                              ({9: ODD}, A), ({6: HALF}, A), ({7: HALF}, A)])
    _empty(L.rtn_norm, ok, 4, (2, 9))
    #     0 dt       1 kind 2 du 3 ld 4 x 5 ldx 6 M 7 C 8 w  9 eps  10 add 11 ld 12 dx 13 ld 14 dw 15 db 16 ws 17 wsb 18 st
    ok = [B.RTN_BF16, 1, FAKE, 64, FAKE, 64, 100, 64, FAKE, f(0), FAKE, 64, OTHER, 64, OTHER, OTHER, FAKE, BIG, None]
    _refuses(L.rtn_norm_backward, ok, [
        ({2: None}, N), ({4: None}, N), ({8: None}, N), ({12: None, 14: None, 15: None}, N), ({0: 2}, U), ({1: 5}, U), ({3: 63}, S), ({5: 63}, S),
        ({11: 63}, S), ({13: 63}, S), ({9: f(-1)}, S), ({6: -1}, S), ({7: 16385}, S), ({2: ODD}, A), ({10: ODD}, A), ({12: ODD}, A), ({14: HALF}, A),
        ({16: FOUR}, A), ({16: None}, W), ({17: L.rtn_norm_backward_workspace_bytes(100, 64, 100) - 1}, W)])


def test_block_norm_refuses(L):  # noqa: F811
    f = C.c_float
    #     0 dt       1 k 2 h 3 ld 4 x 5 ld 6 M 7 C 8 w  9 b   10 gate 11 run 12 scale 13 nw 14 nb 15 eps 16 y 17 ld 18 u 19 ld 20 st
    ok = [B.RTN_BF16, 0, FAKE, 64, FAKE, 64, 100, 64, FAKE, FAKE, FAKE, 10, f(1), FAKE, FAKE, f(1e-6), OTHER, 64, OTHER, 64, None]
    _refuses(L.rtn_block_norm, ok, [
        ({2: None}, N), ({4: None}, N), ({8: None}, N), ({13: None}, N), ({16: None}, N), ({0: 2}, U), ({1: 2}, U), ({3: 63}, S), ({5: 63}, S), ({17: 63}, S),
        ({19: 63}, S), ({11: 0}, S), ({11: -3}, S), ({15: f(-1)}, S), ({7: 16385}, S), ({2: ODD}, A), ({4: ODD}, A), ({16: ODD}, A), ({18: ODD}, A),
        ({10: HALF}, A), ({13: HALF}, A), ({14: HALF}, A)])
    _empty(L.rtn_block_norm, ok, 6, (2, 4, 16))
    #     0 dt       1 k 2 dy 3 ld 4 du 5 ld 6 h 7 ld 8 y 9 ld 10 M 11 C 12 w 13 b  14 gate 15 run 16 scale 17 nw 18 eps
    ok = [B.RTN_BF16, 0, FAKE, 64, FAKE, 64, FAKE, 64, FAKE, 64, 100, 64, FAKE, FAKE, FAKE, 10, f(1), FAKE, f(1e-6),
          OTHER, 64, OTHER, 64, OTHER, OTHER, OTHER, OTHER, OTHER, FAKE, BIG, None]
    #     19 dh 20 ld 21 dx 22 ld 23 dw 24 db 25 dgate 26 dnw 27 dnb 28 ws 29 wsb 30 st
    _refuses(L.rtn_block_norm_backward, ok, [
        ({2: None, 4: None}, N), ({6: None}, N), ({8: None}, N), ({12: None}, N), ({17: None}, N), ({4: None}, N), ({14: None}, N),
        ({i: None for i in (19, 21, 23, 24, 25, 26, 27)}, N), ({0: 2}, U), ({1: 2}, U), ({3: 63}, S), ({5: 63}, S), ({7: 63}, S), ({9: 63}, S),
        ({20: 63}, S), ({22: 63}, S), ({15: 0}, S), ({18: f(np.nan)}, S), ({10: -1}, S), ({2: ODD}, A), ({8: ODD}, A), ({19: ODD}, A), ({23: HALF}, A),
        ({25: HALF}, A), ({28: FOUR}, A), ({28: None}, W), ({29: L.rtn_norm_backward_workspace_bytes(100, 64, 10) - 1}, W)])


def test_units_of_the_norms_gradients_fill_whole_rounds(L):  # noqa: F811
    """The units of all rows of the gate, which the workspace holds four sums of each for (and four of each of up to 64 blocks of owners), are no
    more than the chip holds at 16 waves to a CU, or one for each owner, or three where those fit twice."""
    rng = np.random.default_rng(1)
    for C, held in ((64, 4096), (512, 4096), (513, 1024), (2048, 1024), (2187, 512), (4096, 512), (4100, 256), (8192, 256), (16384, 256)):
        for M in [1, 2, 255, 256, 300, 1000, 2000, 16384] + [int(m) for m in np.exp(rng.uniform(0, np.log(1 << 20), 30))]:
            for G in [1, 2, 3, 5, 7, 24, 100, 255, 256, 257, 300] + [int(g) for g in np.exp(rng.uniform(0, np.log(M + 1), 30))]:
                run = -(-M // min(G, M))
                owners = -(-M // run)
                units, rest = divmod(L.rtn_norm_backward_workspace_bytes(M, C, run), 16 * C)
                units -= min(owners, 64)
                assert rest == 0 and units % owners == 0 and units > 0, (M, C, run, units)
                assert units <= held or units == owners or units <= 3 * owners < 2 * held < 4 * owners, (M, C, run, units)


@pytest.mark.parametrize("call", [lambda t: B.mx4_pack(t), lambda t: B.mx4_linear(t, t, 4), lambda t: B.norm(t, t[0]), lambda t: B.block_norm(t, t, t[0])])
def test_the_binding_takes_device_tensors_only(call):
    import torch
    with pytest.raises(AssertionError):
        call(torch.zeros((4, 4), dtype=torch.bfloat16))


def test_sizes_of_the_tests_reach_every_form(tmp_path):
    """Every form of the product, and tiles with edges inside, over fewer, as many and more steps of 128 columns than their ring holds."""
    import test_mx4_linear as G
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_02057_amd", "csrc")
    (tmp_path / "r.cpp").write_text("""#include "choice.h"
extern "C" int form(int64_t M, int64_t N, int64_t K) { return (int)rtn::mx4_form(M, N, K); }
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + csrc, str(tmp_path / "r.cpp"), "-o", str(tmp_path / "r.so")], check=True)
    form = C.CDLL(str(tmp_path / "r.so")).form
    form.argtypes = [C.c_int64] * 3
    sizes = G.SIZES + G.TILES
    assert {form(*s) for s in sizes} == set(range(9))
    for f, ring in ((6, 4), (7, 3), (8, 4)):
        steps = [-(-K // 128) for M, N, K in sizes if form(M, N, K) == f]
        assert min(steps) == 1 and max(steps) > ring + 1 and any(M % 128 and N % 128 for M, N, K in sizes if form(M, N, K) == f), (f, steps)


def test_sizes_of_the_gradients_reach_the_larger_forms(tmp_path):
    """dx is a product of M x K over N, dw, whose sums may leave in fp32, of N x K over M: each in all forms from the 64 x 64 blocks of four
    waves on, with edges inside the tiles; and the forward pass' epilogues and pitches."""
    import test_mx4_linear as G
    csrc = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_1912_02057_amd", "csrc")
    (tmp_path / "r.cpp").write_text("""#include "choice.h"
extern "C" int form(int64_t M, int64_t N, int64_t K) { return (int)rtn::mx4_form(M, N, K); }
""")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-shared", "-fPIC", "-I" + csrc, str(tmp_path / "r.cpp"), "-o", str(tmp_path / "r.so")], check=True)
    form = C.CDLL(str(tmp_path / "r.so")).form
    form.argtypes = [C.c_int64] * 3
    dx, dw = [(M, K, N) for M, N, K in G.GRADS], [(N, K, M) for M, N, K in G.GRADS]
    for sizes in (dx, dw, G.FORMS):
        for f in (5, 6, 7, 8):
            assert any(form(*s) == f and s[0] % 128 and s[1] % 128 for s in sizes), (f, sizes)
    assert any(form(*s) == 8 and s[0] % 256 == 0 == s[1] % 256 for s in dw)
    assert any(form(*s) in (6, 7, 8) and s[2] > 5 * 128 for s in dx) and any(form(*s) in (6, 7, 8) and s[2] > 5 * 128 for s in dw)
    assert any(form(*s) == 7 and s[0] * s[1] >= 1 << 25 for s in G.FORMS)
