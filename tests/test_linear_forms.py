"""Sizes that reach every form of the linear layer's kernels, with odd edges: the tiles over many steps, rows that are copied first, each tile of
the weight gradient with and without its tokens split, and sums of dz over runs of several blocks.  (test_linear_forms_cpu.py checks on
the host that they do.)  Against plain 64-bit forms on the device."""
import math

import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu

# M, N, K, first column of x within its rows: odd columns and shifted starts are copied for tiles and for long rows
FORWARD = [(1100, 1000, 2003, 0), (1100, 1000, 2008, 0), (1030, 1100, 333, 1), (2300, 2100, 333, 0), (2300, 2100, 328, 0), (2211, 2091, 328, 1),
           (2300, 2100, 1000, 0), (216, 600, 4223, 0), (33, 300, 4160, 1), (500, 1500, 4187, 3), (250, 1300, 4187, 0), (400, 1500, 2600, 0), (70, 1030, 2187, 0)]
# M, N, K of a backward pass: tiles of 128 over 1, 2, 3 and more steps of 64 tokens, of 256, and both and 64 with the tokens split
BACKWARD = [(33, 724, 5600), (100, 730, 5601), (130, 724, 5600), (200, 727, 5603), (5000, 70, 5600), (6001, 250, 3001), (300, 2208, 5388), (515, 1030, 7687),
            (17000, 136, 5600), (6000, 1030, 4100), (1100, 131, 1500), (4500, 129, 133), (2112, 66, 64), (17000, 2100, 40), (16500, 8200, 16)]


def double(t):
    return t.double()


def act64(z, name):
    if name == "relu":
        return z.clamp_min(0)
    if name == "gelu":
        return z * torch.special.ndtr(z)
    return z * torch.sigmoid(z) if name == "silu" else z


def slope64(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


class Case:
    def __init__(self, dtype, M, N, K, start=0, vector=True):
        self.dtype, self.type, self.M, self.N, self.K = dtype, T.TYPES[dtype], M, N, K
        g = torch.Generator(device=T.DEV)
        g.manual_seed(M + 3 * N + 7 * K + start)
        rand = lambda *s: torch.randn(s, generator=g, device=T.DEV)
        self.t = torch.randint(-1, 2, (N, K), generator=g, device=T.DEV, dtype=torch.int8)
        self.codes = torch.zeros((N, -(-K // 64) * 64), dtype=torch.int8, device=T.DEV)
        self.codes[:, :K] = self.t
        x = torch.full((M, K + start), float("nan"), dtype=self.type, device=T.DEV)
        x[:, start:] = (rand(M, K) * torch.exp(0.5 * rand(K))).to(self.type)
        self.x, self.dy = x[:, start:], rand(M, N).to(self.type)
        self.bias, self.res = (0.3 * rand(N)).to(self.type), rand(M, N).to(self.type)
        self.alpha = (0.5 + torch.rand(N, generator=g, device=T.DEV)) / math.sqrt(K) if vector else 1.25 / math.sqrt(K)

    def rounded(self, v, e):
        return T.U[self.dtype] * (v.abs() + e) + e + T.STEP[self.dtype]


def within(got, want, bound, what):
    off = (got.double() - want).abs()
    bad = ~(off <= bound)
    assert got.shape == want.shape and not bad.any(), (what, int(bad.sum()), float(off[bad].max()), bad.nonzero()[0].tolist())


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", FORWARD)
def test_forward_forms(dtype, size):
    M, N, K, start = size
    print("[case] linear forward", dtype, size, flush=True)
    c = Case(dtype, M, N, K, start)
    w = B.linear_prepare(c.codes, N, K)
    t, a, b = double(c.t), double(c.alpha), double(c.bias)
    z = torch.matmul(double(c.x), t.t().contiguous()) * a + b
    ez = (K + 3) * T.EPS * (torch.matmul(double(c.x).abs(), t.abs().t().contiguous()) * a + b.abs())
    for name in ("none", "relu", "gelu", "silu"):
        y = act64(z, name)
        e = 1.13 * ez + (T.ACT_EPS * z.abs().clamp_min(1) if name in ("gelu", "silu") else 0)
        y, e = y + double(c.res), e + T.EPS * (y.abs() + double(c.res).abs())
        kw = dict(bias=c.bias, act=T.ACTS[name], residual=c.res)
        within(B.linear(c.x, w, N, c.alpha, **kw), y, c.rounded(y, e), "y, %s" % name)
        z8 = B.checkpoint_empty(M, N, T.DEV)
        within(B.linear(c.x, w, N, c.alpha, z_ckpt=z8, **kw), y, c.rounded(y, e), "y with a checkpoint, %s" % name)
    zhat = double(B.checkpoint_unpack(z8, M, N, c.type))
    # the step of a group is at most 1/64 of its largest magnitude; a whole one where that lies on the border of two
    top = torch.nn.functional.pad(z.abs(), (0, 0, 0, -M % 32)).view(-1, 32, N).amax(1).repeat_interleave(32, 0)[:M]
    within(zhat, z, top / 64 * (1 + 1e-9) + 2 * ez + 2.0 ** -24, "z^")
    again = B.checkpoint_empty(M, N, T.DEV)
    B.linear(c.x, w, N, c.alpha, z_ckpt=again, **kw)
    assert torch.equal(B.checkpoint_unpack(again, M, N, c.type), zhat.to(c.type))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", BACKWARD)
def test_backward_forms(dtype, size):
    M, N, K = size
    print("[case] linear backward", dtype, size, flush=True)
    for name in ("none", "silu"):
        c = Case(dtype, M, N, K, vector=name == "none")
        wt = B.linear_prepare(c.codes, N, K, backward=True)[1]
        x8 = B.checkpoint_pack(c.x)
        xhat = double(B.checkpoint_unpack(x8, M, K, c.type))
        dy, a, t, u = double(c.dy), c.alpha if name == "silu" else double(c.alpha), double(c.t), T.U[dtype]
        z8, dz, ez = None, dy, torch.zeros_like(dy)
        if name != "none":                                   # any values of z
            z8 = B.checkpoint_pack(c.res)
            z = double(B.checkpoint_unpack(z8, M, N, c.type))
            dz, ez = dy * slope64(z, name), dy.abs() * T.ACT_EPS * z.abs().clamp_min(1)
        # what of a term can be lost below float16's normal values (test_linear_small_gradients.py)
        D, A = float(dy.abs().max()), float(c.alpha) if name == "silu" else float(a.max())
        low = D if dtype == "fp16" else 0.0
        dx = torch.matmul(dz * a, t)
        ex = torch.matmul(ez * a, t.abs()) * (1 + u) + (u + (N + 3) * T.EPS) * torch.matmul((dz * a).abs(), t.abs()) + N * 2.0 ** -38 * low * A
        dw = torch.matmul(dz.t().contiguous(), xhat)
        ew = torch.matmul(ez.t().contiguous(), xhat.abs()) * (1 + u) + ((u if name != "none" else 0.0) + (M + 3) * T.EPS) * torch.matmul(dz.abs().t().contiguous(), xhat.abs())
        ew = ew + 2.0 ** -39 * low * xhat.abs().sum(0)
        db, eb = dz.sum(0), ez.sum(0) + (M + 3) * T.EPS * dz.abs().sum(0)
        kw = dict(act=T.ACTS[name], z_ckpt=z8)
        got = B.linear_backward(c.dy, wt, K, c.alpha, x8, **kw)
        within(got[0], dx, c.rounded(dx, ex), "dx, %s" % name)
        within(got[1], dw, c.rounded(dw, ew), "dw, %s" % name)
        within(got[2], db, c.rounded(db, eb), "dbias, %s" % name)
        f32 = B.linear_backward(c.dy, wt, K, c.alpha, x8, dw_dtype=torch.float32, **kw)
        within(f32[1], dw, ew, "dw in fp32, %s" % name)
        assert torch.equal(f32[0], got[0]) and torch.equal(f32[2], got[2])
        again = B.linear_backward(c.dy, wt, K, c.alpha, x8, **kw)
        assert all(torch.equal(p, q) for p, q in zip(got, again))
        only = B.linear_backward(c.dy, None, K, c.alpha, x8, want_dx=False, want_dbias=False, **kw)
        assert torch.equal(only[1], got[1])


def whole(c, top, *shape):
    """Whole numbers up to `top` in magnitude."""
    return torch.randint(-top, top + 1, shape, device=T.DEV).to(c.type)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", FORWARD)
def test_forward_forms_exactly(dtype, size):
    """Whole numbers and powers of two, whose sums fp32 holds exactly in any order: y is the sum rounded once, to the bit."""
    M, N, K, start = size
    print("[case] linear forward, whole numbers", dtype, size, flush=True)
    c = Case(dtype, M, N, K, start)
    c.x.copy_(whole(c, 15, M, K))
    bias, res = whole(c, 15, N) / 8, whole(c, 15, M, N) / 8
    alpha = torch.exp2(-torch.randint(1, 5, (N,), device=T.DEV).float())
    z = torch.matmul(double(c.x), double(c.t).t().contiguous()) * double(alpha) + double(bias)
    w = B.linear_prepare(c.codes, N, K)
    for name in ("none", "relu"):
        want = (act64(z, name) + double(res)).to(c.type)
        z8 = B.checkpoint_empty(M, N, T.DEV)
        for kw in (dict(), dict(z_ckpt=z8)):
            assert torch.equal(B.linear(c.x, w, N, alpha, bias=bias, act=T.ACTS[name], residual=res, **kw), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", BACKWARD)
def test_backward_forms_exactly(dtype, size):
    """The same for the gradients: no token, channel or split is left out or counted twice."""
    M, N, K = size
    print("[case] linear backward, whole numbers", dtype, size, flush=True)
    c = Case(dtype, M, N, K)
    c.x.copy_(whole(c, 15, M, K))                            # exact in a checkpoint
    dy, t = whole(c, 3, M, N), double(c.t)
    wt = B.linear_prepare(c.codes, N, K, backward=True)[1]
    x8, z8 = B.checkpoint_pack(c.x), B.checkpoint_pack(c.res)
    for name, alpha in (("none", 0.25), ("relu", torch.exp2(-torch.randint(1, 5, (N,), device=T.DEV).float()))):
        dz = double(dy) * (1 if name == "none" else slope64(double(B.checkpoint_unpack(z8, M, N, c.type)), name))
        dx = torch.matmul(dz * (double(alpha) if torch.is_tensor(alpha) else alpha), t)
        dw = torch.matmul(dz.t().contiguous(), double(c.x))
        kw = dict(act=T.ACTS[name], z_ckpt=z8 if name != "none" else None)
        got = B.linear_backward(dy, wt, K, alpha, x8, **kw)
        assert torch.equal(got[0], dx.to(c.type)) and torch.equal(got[1], dw.to(c.type)) and torch.equal(got[2], dz.sum(0).to(c.type))
        assert torch.equal(B.linear_backward(dy, None, K, alpha, x8, want_dx=False, want_dbias=False, dw_dtype=torch.float32, **kw)[1], dw.float())
