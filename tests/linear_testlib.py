"""Plain 64-bit forms (numpy) of the ternary linear layer and of the 8-bit checkpoints, and the bounds that the
library's results are held to.

Bounds.  u is the unit roundoff of the 16-bit type (2^-8 bfloat16, 2^-11 float16) and eps = 2^-24 that of fp32.  A sum of n
fp32 terms in any order is off by at most n eps times the sum of their magnitudes; the activations and slopes are evaluated in
fp32, within ACT_EPS = 2^-19 of max(1, |z|) (erf, exp and the products around them: some ten roundings, and exp's argument is rounded
relative to itself), and change by at most 1.13 resp. 1.2 times a change of z (the largest slopes of gelu and silu and of
their slopes).  An output is rounded once: u |y|, or half the least subnormal step."""
import math

import numpy as np
import torch

from paper_1912_02057_amd import binding as B

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
STEP = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -24}
LEAST, MOST = {"bf16": -126, "fp16": -24}, {"bf16": 121, "fp16": 9}
ACTS = {"none": B.RTN_ACT_NONE, "relu": B.RTN_ACT_RELU, "gelu": B.RTN_ACT_GELU, "silu": B.RTN_ACT_SILU}
EPS, ACT_EPS = 2.0 ** -24, 2.0 ** -19
_erf = np.vectorize(math.erf, otypes=[np.float64])


def f64(t):
    return t.detach().double().cpu().numpy()


def act(z, name):
    if name == "relu":
        return np.where(z > 0, z, np.where(np.isnan(z), z, 0.0))
    if name == "gelu":
        return 0.5 * z * (1 + _erf(z / math.sqrt(2)))
    if name == "silu":
        with np.errstate(over="ignore"):
            return z / (1 + np.exp(-z))
    return z


def slope(z, name):
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return np.where(z > 0, 1.0, 0.0)
    if name == "gelu":
        return 0.5 * (1 + _erf(z / math.sqrt(2))) + z * np.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    with np.errstate(over="ignore"):
        s = 1 / (1 + np.exp(-z))
    return s * (1 + z * (1 - s))


def eight_bits(v, dtype):
    """(v^, 2^e of every element) of the 8-bit checkpoint of v, in 64 bits."""
    out, scale = np.empty_like(v), np.empty_like(v)
    for i in range(0, v.shape[0], 32):
        p = v[i:i + 32]
        a = np.abs(p).max(axis=0)
        ok = np.isfinite(a)
        e = np.frexp(np.where(ok & (a > 0), a, 1.0))[1] - 7
        e = np.where(np.rint(np.ldexp(np.where(ok, a, 0.0), -e)) > 127, e + 1, e)
        e = np.clip(np.where(a > 0, e, -10000), LEAST[dtype], MOST[dtype])
        s = np.ldexp(1.0, e)
        with np.errstate(invalid="ignore"):
            out[i:i + 32] = np.where(ok, np.clip(np.rint(p / s), -127, 127) * s, np.nan)
        scale[i:i + 32] = s
    return out, scale


def codes_of(t, fmt=B.RTN_CODE_I8):
    """Ternary matrix (numpy int8) -> device codes as ternarize_pack writes them."""
    return B.ternarize_pack(torch.from_numpy(t.astype(np.float32)).to(DEV), -0.5, 0.5, fmt, want_sum=False)[0]


class Layer:
    """Inputs of one layer, on the device and in 64 bits."""

    def __init__(self, dtype, M, N, K, seed, bias=True, residual=True, vector=True, zeros=1 / 3):
        rng = np.random.default_rng(seed)
        self.dtype, self.type, self.M, self.N, self.K = dtype, TYPES[dtype], M, N, K
        dev = lambda a: torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(DEV)
        half = lambda a: dev(a).to(self.type)
        self.t = (rng.random((N, K)) >= zeros) * rng.choice([-1, 1], (N, K))
        channel = np.exp(0.5 * rng.standard_normal(K)) * np.where(rng.random(K) < 0.02, 20, 1)
        self.x = half(rng.standard_normal((M, K)) * channel)
        self.dy = half(rng.standard_normal((M, N)))
        self.alpha = dev((0.5 + rng.random(N)) / math.sqrt(K)) if vector else float(np.float32(1.3 / math.sqrt(K)))
        self.bias = half(0.3 * rng.standard_normal(N)) if bias else None
        self.res = half(rng.standard_normal((M, N))) if residual else None
        self.codes = codes_of(self.t)

    @property
    def a64(self):
        return f64(self.alpha) if torch.is_tensor(self.alpha) else np.full(self.N, self.alpha)

    def z64(self):
        """z and a bound of the error of its fp32 evaluation."""
        x, a = f64(self.x), self.a64
        b = f64(self.bias) if self.bias is not None else np.zeros(self.N)
        z = (x @ self.t.T) * a + b
        return z, (self.K + 3) * EPS * ((np.abs(x) @ np.abs(self.t).T) * np.abs(a) + np.abs(b))

    def y64(self, name):
        z, ez = self.z64()
        y = act(z, name)
        ey = 1.13 * ez + (ACT_EPS * np.maximum(1, np.abs(z)) if name in ("gelu", "silu") else 0)
        if self.res is not None:
            r = f64(self.res)
            y, ey = y + r, ey + EPS * (np.abs(y) + np.abs(r))
        return y, ey

    def rounded(self, v, e):
        """The bound of a 16-bit output of value v whose fp32 form is off by e."""
        return U[self.dtype] * (np.abs(v) + e) + e + STEP[self.dtype]

    def grads64(self, name, xhat, zhat):
        """dx, dw, dbias from the values that the checkpoints stand for, and their fp32 bounds."""
        dy, a, u = f64(self.dy), self.a64, U[self.dtype]
        s = slope(zhat, name) if name != "none" else np.ones_like(dy)
        zhat = np.zeros_like(dy) if zhat is None else zhat
        dz = dy * s
        ez = np.abs(dy) * (ACT_EPS * np.maximum(1, np.abs(zhat)) if name in ("gelu", "silu") else 0)
        ru = u if name != "none" else 0.0                   # dz is dy itself without an activation
        rx = u if name != "none" or torch.is_tensor(self.alpha) else 0.0
        sx = (np.abs(dz * a)) @ np.abs(self.t)
        dx = (dz * a) @ self.t
        ex = (ez * np.abs(a)) @ np.abs(self.t) * (1 + u) + (rx + (self.N + 3) * EPS) * sx + self.N * STEP[self.dtype]
        sw = np.abs(dz).T @ np.abs(xhat)
        dw = dz.T @ xhat
        ew = ez.T @ np.abs(xhat) * (1 + u) + (ru + (self.M + 3) * EPS) * sw + STEP[self.dtype] * np.abs(xhat).sum(0)
        return (dx, ex), (dw, ew), (dz.sum(0), ez.sum(0) + (self.M + 3) * EPS * np.abs(dz).sum(0))


def assert_within(got, want, bound, what):
    got = f64(got) if torch.is_tensor(got) else got
    assert got.shape == want.shape, (what, got.shape, want.shape)
    off = np.abs(got - want)
    bad = ~(off <= bound)
    assert not bad.any(), "%s: %d of %d off, worst %g over its bound %g at %s" % (
        what, bad.sum(), bad.size, np.nanmax(np.where(bad, off, 0)), bound.flat[int(np.argmax(np.where(bad, off, 0)))],
        np.unravel_index(int(np.argmax(np.where(bad, off, 0))), bad.shape))
