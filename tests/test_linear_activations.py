"""GELU and its slope over the whole range, tails included, to a relative 2^-15 and one rounding: z is x itself here (one input,
weight +1, alpha 1).

Bounds.  The normal tail Q is fitted to 2^-15.8 of itself; exp(-z^2 / 2) has its argument rounded relative to itself, 2^-23 z^2 / 2 (2^-16.6
at |z| = 13.2, where exp is 2^-126); the products around them are some ten roundings of 2^-24.  Together below 2^-15 of Q, and of
z times the density.  Values below 2^-120 may come out as zero, since exp2 gives no subnormal numbers."""
import numpy as np
import pytest
import torch
from scipy.special import ndtr

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu
REL, LEAST = 2.0 ** -15, 2.0 ** -120


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_gelu_in_its_tails(dtype):
    z = np.concatenate([np.linspace(-14, 14, 4001), -np.exp2(np.linspace(-20, 6, 500)), [0.0, -0.0]])
    x = torch.from_numpy(z).to(T.TYPES[dtype]).to(T.DEV)[:, None].contiguous()
    z = T.f64(x)
    w = B.linear_prepare(T.codes_of(np.ones((1, 1))), 1, 1)
    y = T.f64(B.linear(x, w, 1, 1.0, act=B.RTN_ACT_GELU))
    want = z * ndtr(z)
    u = T.U[dtype]
    T.assert_within(y, want, np.abs(want) * (REL + u * (1 + REL)) + LEAST + T.STEP[dtype], "gelu")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_slope_of_gelu_in_its_tails(dtype):
    """dbias of one token is the slope (dy = 1)."""
    N = 3000
    z = np.linspace(-14, 14, N)
    bias = torch.from_numpy(z).to(T.TYPES[dtype]).to(T.DEV)
    codes = T.codes_of(np.zeros((N, 1)))
    x = torch.zeros((1, 1), dtype=T.TYPES[dtype], device=T.DEV)
    z8 = B.checkpoint_empty(1, N, T.DEV)
    B.linear(x, B.linear_prepare(codes, N, 1), N, 1.0, bias=bias, act=B.RTN_ACT_GELU, z_ckpt=z8)
    zhat = T.f64(B.checkpoint_unpack(z8, 1, N, T.TYPES[dtype]))[0]
    dy = torch.ones((1, N), dtype=T.TYPES[dtype], device=T.DEV)
    got = T.f64(B.linear_backward(dy, None, 1, 1.0, None, act=B.RTN_ACT_GELU, z_ckpt=z8, want_dx=False, want_dw=False)[2])
    phi, density = ndtr(zhat), zhat * np.exp(-zhat ** 2 / 2) / np.sqrt(2 * np.pi)
    want, u = phi + density, T.U[dtype]
    off = REL * (phi + np.abs(density))
    T.assert_within(got, want, off + u * (np.abs(want) + off) + LEAST + T.STEP[dtype], "slope")
