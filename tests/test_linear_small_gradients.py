"""float16 gradients whose size is far from 1, and that of alpha too: every term of dx and dw keeps its 11 bits.

Bounds.  A term of dx is dz alpha t, of dw dz x^, with dz alpha resp. dz rounded to float16 relative to a power of two that
brings the largest of them to 2^13 or above.  So a term is off by u of itself, or, where its operand falls below the normal values, by
2^-25 in a unit of at most 2^-13 D A resp. 2^-14 D, with D = max |dy| and A = max |alpha|: less than 2^-38 D A resp. 2^-39 D."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu


def bounds(L, name, xhat, zhat):
    """grads64 with the terms' subnormal steps replaced by the bounds above."""
    (dx, ex), (dw, ew), db = L.grads64(name, xhat, zhat)
    D, A, step = np.abs(T.f64(L.dy)).max(), np.abs(L.a64).max(), T.STEP["fp16"]
    columns = np.abs(xhat).sum(0)
    return (dx, ex - L.N * step + L.N * 2.0 ** -38 * D * A), (dw, ew - step * columns + 2.0 ** -39 * D * columns), db


# dx by the kernels for a few tokens, small grids and tiles
@pytest.mark.parametrize("size", [(3, 96, 200), (40, 640, 333), (1100, 600, 1000)])
@pytest.mark.parametrize("vector", [False, True])
@pytest.mark.parametrize("scale", [1e-4, 1e-5, 1e-6, 1.2e4])
def test_every_term_keeps_its_bits(size, vector, scale):
    M, N, K = size
    print("[case] float16 gradients", size, vector, scale, flush=True)
    L = T.Layer("fp16", M, N, K, seed=M + N, residual=False, vector=vector)
    rng = np.random.default_rng(M)
    dy = scale * rng.standard_normal((M, N))
    if scale > 1:                                            # up to the type's end, where dz alone would be infinite
        dy[:, ::7] = rng.choice([-65000.0, 65000.0], dy[:, ::7].shape)
        L.alpha = 0.1 * L.alpha
        if not vector:
            L.alpha = float(np.float32(L.alpha))
    L.dy = torch.from_numpy(dy).to(torch.float16).to(T.DEV)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    x8 = B.checkpoint_pack(L.x)
    xhat = T.f64(B.checkpoint_unpack(x8, M, K, L.type))
    for name in ("none", "relu", "gelu", "silu"):
        z8, zhat = None, np.zeros((M, N))
        if name != "none":
            z8 = B.checkpoint_empty(M, N, T.DEV)
            B.linear(L.x, w, N, L.alpha, bias=L.bias, act=T.ACTS[name], z_ckpt=z8)
            zhat = T.f64(B.checkpoint_unpack(z8, M, N, L.type))
        (dx, ex), (dw, ew), _ = bounds(L, name, xhat, zhat)
        got = B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS[name], z_ckpt=z8, want_dbias=False, dw_dtype=torch.float32)
        T.assert_within(got[0], dx, L.rounded(dx, ex), "dx, %s" % name)
        T.assert_within(got[1], dw, ew, "dw, %s" % name)
        only = B.linear_backward(L.dy, wt, K, L.alpha, None, act=T.ACTS[name], z_ckpt=z8, want_dw=False, want_dbias=False)
        assert torch.equal(only[0], got[0])
        only = B.linear_backward(L.dy, None, K, L.alpha, x8, act=T.ACTS[name], z_ckpt=z8, want_dx=False, want_dbias=False, dw_dtype=torch.float32)
        assert torch.equal(only[1], got[1])


@pytest.mark.parametrize("M", [4, 70])
def test_scales_at_their_ends(M):
    """All of dy zero, one element the only one, alpha zero, tiny or huge, and infinities and NaNs in dy, which stay in their rows
    of dx and columns of dw."""
    N, K = 48, 136
    L = T.Layer("fp16", M, N, K, seed=7)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    x8, z8 = B.checkpoint_pack(L.x), B.checkpoint_empty(M, N, T.DEV)
    B.linear(L.x, w, N, L.alpha, bias=L.bias, act=T.ACTS["gelu"], z_ckpt=z8)
    xhat, zhat = (T.f64(B.checkpoint_unpack(c, M, n, L.type)) for c, n in ((x8, K), (z8, N)))
    call = lambda: B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS["gelu"], z_ckpt=z8, dw_dtype=torch.float32)
    ones, first = L.alpha.clone(), L.dy.clone()

    def check():
        (dx, ex), (dw, ew), _ = bounds(L, "gelu", xhat, zhat)
        got = call()
        T.assert_within(got[0], dx, L.rounded(dx, ex), "dx")
        T.assert_within(got[1], dw, ew, "dw")
    for alpha in (2.0 ** -60, 2.0 ** -126, 2.0 ** 20):
        L.alpha, L.dy = ones * alpha, first if alpha < 1 else first * 2.0 ** -20
        check()
    L.alpha, L.dy = ones, torch.zeros_like(first)
    assert all(not g.any() for g in call())
    L.dy[M - 1, N - 1] = 2.0 ** -24
    check()
    L.alpha, L.dy = torch.zeros_like(ones), first
    assert not call()[0].any()
    L.alpha, L.dy = ones, first.clone()
    L.dy[1, 5], L.dy[M - 1, 40] = float("inf"), float("nan")
    dx, dw, db = (T.f64(g) for g in call())
    keep, rows = [m for m in range(M) if m not in (1, M - 1)], [n for n in range(N) if n not in (5, 40)]
    L.dy[1], L.dy[M - 1] = 0, 0
    (want, ex), _, _ = L.grads64("gelu", xhat, zhat)          # terms with the subnormal steps of the unscaled type
    T.assert_within(dx[keep], want[keep], L.rounded(want, ex)[keep], "dx")
    assert not np.isfinite(dx[[1, M - 1]]).any() and np.isfinite(dw[rows]).all() and not np.isfinite(dw[[5, 40]]).any()


def test_units_follow_the_data_of_a_replay():
    """A recorded backward pass takes its powers of two from the dy and alpha of each replay."""
    M, N, K = 96, 200, 136
    L = T.Layer("fp16", M, N, K, seed=3)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    x8, z8 = B.checkpoint_pack(L.x), B.checkpoint_empty(M, N, T.DEV)
    B.linear(L.x, w, N, L.alpha, bias=L.bias, act=T.ACTS["gelu"], z_ckpt=z8)
    dy, alpha = L.dy.clone(), L.alpha.clone()
    ws = torch.empty(B.lib().rtn_linear_backward_workspace_bytes(M, N, K), dtype=torch.uint8, device=T.DEV)
    call = lambda **kw: B.linear_backward(dy, wt, K, alpha, x8, act=T.ACTS["gelu"], z_ckpt=z8, **kw)
    dx, dw, db = call(workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(dx=dx, dw=dw, dbias=db, workspace=ws)
    for size in (1.0, 1e-5, 3e3, 1e-3):
        dy.copy_(L.dy * size)
        alpha.copy_(L.alpha * size ** 0.5)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), call()))
