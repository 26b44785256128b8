"""Microscaled 4-bit packing against its definition in 64 bits, exactly."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import mx4_testlib as Q
from mx4_testlib import collected  # noqa: F401 (a fixture of the module)

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (1, 32), (3, 31), (16, 128), (17, 129), (64, 33), (65, 512), (77, 1000), (130, 257), (300, 96)]


def check(x, seed, both=True):
    R, C = x.shape
    s = Q.seed_tensor(seed)
    with np.errstate(over="ignore"):                           # (the largest finite values may round to 4 x 2^126, infinite in fp32)
        want, want_t = [v.astype(np.float32).astype(np.float64) for v in (Q.four(Q.f64(x), seed), Q.four(Q.f64(x).T, seed, True))]
    if both:
        p, pt = B.mx4_pack(x, seed=s, transposed=True)
        Q.equal(B.mx4_unpack(pt, C, R, torch.float32), want_t)
    else:
        p = B.mx4_pack(x, seed=s)
    Q.equal(B.mx4_unpack(p, R, C, torch.float32), want)
    return p, want


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("seed", [None, 12345, -7])
@pytest.mark.parametrize("R,C", SIZES)
def test_values(dtype, seed, R, C):
    x = Q.values(np.random.default_rng(R * 1000 + C), R, C, dtype)
    p, want = check(x, seed, both=False)
    p2, _ = check(x, seed, both=True)
    assert torch.equal(p, p2)                                  # the packing of the rows is the same alone and with the other
    # values of a 16-bit type read back exactly in it
    if dtype != "fp32":
        Q.equal(B.mx4_unpack(p, R, C, Q.TYPES[dtype]), want)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_apart(dtype):
    x = Q.values(np.random.default_rng(3), 70, 205, dtype)
    view = Q.apart(x)
    for seed in (None, 99):
        s = Q.seed_tensor(seed)
        for a, b in zip(B.mx4_pack(x, seed=s, transposed=True), B.mx4_pack(view, seed=s, transposed=True)):
            assert torch.equal(a, b)
        assert torch.equal(B.mx4_pack(x, seed=s), B.mx4_pack(view, seed=s))
    out = Q.apart(torch.zeros((70, 205), dtype=x.dtype, device=Q.DEV))
    p = B.mx4_pack(x)
    B.mx4_unpack(p, 70, 205, x.dtype, out=out)
    assert torch.equal(out, B.mx4_unpack(p, 70, 205, x.dtype))
    assert (out._base.view(-1)[1:].view(70, 208)[:, 205:] == 7).all()   # between the rows nothing is written


@pytest.mark.parametrize("seed", [None, 5])
def test_borders_and_ties(seed):
    """Every multiple of 1/16 of a unit up to 8, with its neighbours in fp32, at scales up to the ends of the range."""
    base = np.arange(0, 129) / 16
    v = np.concatenate([base, np.nextafter(base.astype(np.float32), np.float32(9)), np.nextafter(base.astype(np.float32), np.float32(0))])
    v = np.concatenate([v, -v]).astype(np.float32)
    for e in (0, 1, -3, 100, 124, -100, -122, -125, -127):
        for top in (4.0, 6.0, 6.5, 7.75):                      # with a largest magnitude that fixes the group's scale
            rows = v[np.abs(v) <= top]
            rows = np.concatenate([rows, np.zeros(-len(rows) % 31)]).reshape(-1, 31)
            with np.errstate(over="ignore"):
                x = np.ldexp(np.concatenate([rows, np.full((len(rows), 1), top)], axis=1), e).astype(np.float32)
            assert np.isfinite(x).all()
            check(torch.from_numpy(x).to(Q.DEV), seed)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("seed", [None, 5])
def test_ends_of_the_types(dtype, seed):
    t = Q.TYPES[dtype]
    info = torch.finfo(t)
    tiny = float(info.smallest_normal) * float(info.eps)       # the least subnormal
    x = torch.zeros((40, 64), device=Q.DEV)
    x[1] = tiny
    x[2, ::2] = -3 * tiny
    x[3] = float(info.max)
    x[4, 0], x[4, 1] = float(info.max), -float(info.max) / 2
    x[5] = float(info.smallest_normal)
    x[6, 33] = float(info.smallest_normal) * 1.5
    x[7, :] = torch.linspace(-1, 1, 64, device=Q.DEV)
    x[8, 5] = -0.0
    check(x.to(t), seed)


@pytest.mark.parametrize("seed", [None, 5])
def test_infinities_and_nan_stay_in_their_groups(seed):
    x = Q.values(np.random.default_rng(4), 50, 100, "bf16")
    x[3, 40], x[7, 99], x[40, 0] = float("inf"), float("nan"), float("-inf")
    _, want = check(x, seed)
    assert np.isnan(want[3, 32:64]).all() and np.isfinite(want[3, :32]).all() and np.isnan(want[7, 96:]).all()
    for dtype in (torch.bfloat16, torch.float16, torch.float32):
        got = B.mx4_unpack(B.mx4_pack(x), 50, 100, dtype)
        assert torch.isnan(got[3, 32:64]).all() and torch.isnan(got[7, 96:]).all()


def test_stochastic_rounding_is_unbiased_and_follows_its_seed():
    x = Q.values(np.random.default_rng(5), 8, 64, "bf16")
    total, n = np.zeros((8, 64)), 256
    for s in range(n):
        total += Q.f64(B.mx4_unpack(B.mx4_pack(x, seed=Q.seed_tensor(1000 + s)), 8, 64, torch.float32))
    # a rounding is off by less than a gap, of which the largest is 2 of a unit >= a / 8: the mean of n within 6 standard deviations of at most
    # half a gap each, and the 2^-17 of a gap that 16 bits are short of
    a = np.abs(Q.f64(x)).reshape(8, 2, 32).max(-1, keepdims=True)
    gap = np.broadcast_to(a / 2, (8, 2, 32)).reshape(8, 64)
    assert (np.abs(total / n - Q.f64(x)) <= gap * (6 * 0.5 / np.sqrt(n) + 2.0 ** -16)).all()
    one, same, other = [B.mx4_pack(x, seed=Q.seed_tensor(s)) for s in (1, 1, 2)]
    assert torch.equal(one, same) and not torch.equal(one, other)
    high = B.mx4_pack(x, seed=Q.seed_tensor(1 + (1 << 40)))    # the high word counts
    assert not torch.equal(one, high)


def test_given_buffers_and_nothing_to_do():
    x = Q.values(np.random.default_rng(6), 20, 50, "bf16")
    p, pt = B.mx4_pack(x, transposed=True)
    size, size_t = B.lib().rtn_mx4_bytes(20, 50), B.lib().rtn_mx4_bytes(50, 20)
    a, b = [torch.full((s + 64,), 9, dtype=torch.uint8, device=Q.DEV) for s in (size, size_t)]
    got = B.mx4_pack(x, packed=a, packed_t=b)
    assert got[0].data_ptr() == a.data_ptr() and got[1].data_ptr() == b.data_ptr()
    assert torch.equal(a[:size], p) and (a[size:] == 9).all() and torch.equal(b[:size_t], pt) and (b[size_t:] == 9).all()
    empty = torch.empty((0, 50), dtype=torch.bfloat16, device=Q.DEV)
    assert B.mx4_pack(empty).numel() == 0
    assert B.mx4_unpack(B.mx4_pack(empty), 0, 50, torch.float16).shape == (0, 50)


def test_more_than_4_gib():
    """Offsets past 32 bits: a matrix of 2^31 + elements, checked at its last rows."""
    R, C = 131072 + 40, 16384
    x = torch.zeros((R, C), dtype=torch.bfloat16, device=Q.DEV)
    tail = Q.values(np.random.default_rng(8), 40, C, "bf16")
    x[-40:] = tail
    p, pt = B.mx4_pack(x, transposed=True)
    assert torch.equal(p, B.mx4_pack(x))
    y = B.mx4_unpack(p, R, C, torch.bfloat16)
    assert not y[:-40].any()
    Q.equal(y[-40:], Q.four(Q.f64(tail)))
    del y, p
    yt = B.mx4_unpack(pt, C, R, torch.bfloat16)
    want = Q.four(np.pad(Q.f64(tail).T, ((0, 0), (0, 24))))[:, :40]     # R - 40 is a multiple of 32: the last groups are of the tail
    assert not yt[:, :-40].any()
    Q.equal(yt[:, -40:], want)
