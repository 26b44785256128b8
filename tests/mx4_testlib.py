"""Plain 64-bit forms (numpy) of the microscaled 4-bit operators, and the bounds that the library's results are held to.

Packings are compared exactly: every step from a value to its code is exact in 64 bits and in the kernels.  A product of two packed
values is exact in fp32, and a sum of n such terms in any order is off by at most n eps times the sum of their magnitudes, eps = 2^-24;
terms below 2^-126 may be lost.  Activations are evaluated as in the ternary layer's tests (linear_testlib)."""
import gc

import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

DEV, U, STEP, EPS, ACT_EPS = T.DEV, T.U, T.STEP, T.EPS, T.ACT_EPS
TYPES = dict(T.TYPES, fp32=torch.float32)
f64 = T.f64
GRID = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


@pytest.fixture(autouse=True, scope="module")
def collected():
    """Tensors in reference cycles (tracebacks, wrapped methods) are freed with the module that made them, not in the midst of a later
    test that looks at the device's memory."""
    yield
    gc.collect()


def philox(c, k):
    """Ten rounds on counters c (four uint64 arrays holding 32-bit words) with the two words k of a key."""
    low = np.uint64(0xFFFFFFFF)
    c = [np.asarray(w, dtype=np.uint64) for w in c]
    for i in range(10):
        k0, k1 = np.uint64((k[0] + i * 0x9E3779B9) & 0xFFFFFFFF), np.uint64((k[1] + i * 0xBB67AE85) & 0xFFFFFFFF)
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ k0, b & low, (a >> np.uint64(32)) ^ c[3] ^ k1, a & low]
    return c


def random16(groups, seed, transposed):
    """The 16-bit numbers of groups 0 .. groups - 1: [groups, 32]."""
    g, j = np.meshgrid(np.arange(groups, dtype=np.uint64), np.arange(4, dtype=np.uint64), indexing="ij")
    seed &= (1 << 64) - 1
    w = philox([g & np.uint64(0xFFFFFFFF), g >> np.uint64(32), j, np.full_like(g, int(transposed))], [seed & 0xFFFFFFFF, seed >> 32])
    w = np.stack(w, -1)                                                    # [groups, j, word]
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], -1).reshape(groups, 32).astype(np.float64)


def four(v, seed=None, transposed=False):
    """What the packing of the rows of v (64 bits) stands for."""
    R, C = v.shape
    n = -(-C // 32)
    full = np.zeros((R, 32 * n))
    full[:, :C] = v
    full = full.reshape(-1, 32)
    a = np.abs(full).max(axis=1, keepdims=True)
    ok = np.isfinite(a)
    p = np.where(ok, full, 0.0)
    a = np.where(ok, a, 0.0)
    e = np.where(a > 0, np.frexp(np.where(a > 0, a, 1.0))[1] - 3, -127)
    e = np.maximum(e, -127)
    if seed is not None:
        e = e + (a > np.ldexp(6.0, e))
    r = np.ldexp(np.abs(p), -e)
    if seed is None:
        i = np.zeros(r.shape, dtype=int)
        for k in range(1, 8):
            mid = (GRID[k - 1] + GRID[k]) / 2
            i += (r > mid) | ((r == mid) & (k % 2 == 0))
        q = GRID[i]
    else:
        i = np.minimum(np.searchsorted(GRID, r, side="right") - 1, 6)
        share = (r - GRID[i]) / (GRID[i + 1] - GRID[i])
        q = np.where(random16(R * n, seed, transposed) < share * 65536, GRID[i + 1], GRID[i])
    out = np.where(ok, np.copysign(np.ldexp(q, e), p), np.nan)
    return out.reshape(R, 32 * n)[:, :C]


def seed_tensor(seed):
    return None if seed is None else torch.tensor([seed], dtype=torch.int64, device=DEV)


def values(rng, R, C, dtype, spread=0.7):
    """Values whose channels differ in scale, on the device."""
    v = rng.standard_normal((R, C)) * np.exp(spread * rng.standard_normal(C))
    return torch.from_numpy(v.astype(np.float32)).to(DEV).to(TYPES[dtype])


def apart(t, extra=3, shift=1):
    """The same matrix with its rows `extra` elements apart, starting `shift` elements into a buffer."""
    buf = torch.full((t.shape[0] * (t.shape[1] + extra) + shift,), 7.0, dtype=t.dtype, device=t.device)
    view = buf[shift:].view(t.shape[0], t.shape[1] + extra)[:, :t.shape[1]]
    view.copy_(t)
    return view


def equal(a, b):
    """Equal values; NaN where the other is NaN."""
    a, b = f64(a) if torch.is_tensor(a) else a, f64(b) if torch.is_tensor(b) else b
    assert a.shape == b.shape, (a.shape, b.shape)
    bad = ~((a == b) | (np.isnan(a) & np.isnan(b)))
    assert not bad.any(), "%d of %d differ, first at %s: %r and %r" % (bad.sum(), bad.size, tuple(np.argwhere(bad)[0]), a[bad][0], b[bad][0])


class Layer:
    def __init__(self, dtype, M, N, K, seed=0, bias=True, residual=True):
        rng = np.random.default_rng(seed)
        self.dtype, self.type, self.M, self.N, self.K = dtype, TYPES[dtype], M, N, K
        self.x = values(rng, M, K, dtype)
        self.w = torch.from_numpy((rng.standard_normal((N, K)) / np.sqrt(K)).astype(np.float32)).to(DEV)
        self.dy = values(rng, M, N, dtype)
        half = lambda v: torch.from_numpy(v.astype(np.float32)).to(DEV).to(self.type)
        self.bias = half(0.3 * rng.standard_normal(N)) if bias else None
        self.res = half(rng.standard_normal((M, N))) if residual else None

    def z64(self):
        """z and a bound of the error of its fp32 evaluation."""
        x, w = four(f64(self.x)), four(f64(self.w))
        b = f64(self.bias) if self.bias is not None else np.zeros(self.N)
        return x @ w.T + b, (self.K + 2) * EPS * (np.abs(x) @ np.abs(w).T + np.abs(b)) + self.K * 2.0 ** -126

    def y64(self, act):
        z, ez = self.z64()
        y = T.act(z, act)
        ey = 1.13 * ez + (ACT_EPS * np.maximum(1, np.abs(z)) if act in ("gelu", "silu") else 0)
        if self.res is not None:
            r = f64(self.res)
            y, ey = y + r, ey + EPS * (np.abs(y) + np.abs(r))
        return y, ey

    def rounded(self, v, e):
        return U[self.dtype] * (np.abs(v) + e) + e + STEP[self.dtype]
