"""The 4-bit linear layer and its gradients against their formulas in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T
import mx4_testlib as Q
from mx4_testlib import collected  # noqa: F401 (a fixture of the module)

pytestmark = pytest.mark.gpu

# (M, N, K): one token, a few, many; sizes around the tiles' and the blocks'
SIZES = [(1, 1, 1), (1, 48, 4096), (1, 4096, 130), (2, 33, 31), (5, 100, 257), (15, 64, 128), (16, 70, 500), (3, 200, 4104), (16, 70, 520), (2, 5000, 904), (17, 16, 129), (24, 300, 1000),
         (33, 65, 96), (64, 64, 640), (100, 130, 2187), (129, 257, 300), (256, 1024, 128), (300, 515, 77), (513, 769, 1100), (130, 2050, 700),
         (1000, 1003, 900), (1, 9000, 140)]
# tiles that end inside the matrix, from one block of columns to more than the ring holds
TILES = [(1800, 1747, 100), (1797, 1800, 900), (3500, 3393, 70), (3489, 3500, 1100), (3490, 3400, 390), (257, 30000, 300), (40000, 200, 390),
         (1700, 1300, 3000), (1290, 1030, 2700), (700, 3300, 1030), (1030, 1290, 2600),
         (1290, 1030, 100), (2900, 2900, 70), (300, 35000, 100), (70000, 200, 390), (300, 35000, 700)]


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,N,K", SIZES)
@pytest.mark.parametrize("act", ["none", "gelu"])
def test_forward(dtype, M, N, K, act):
    L = Q.Layer(dtype, M, N, K, seed=M + N + K)
    w = B.mx4_pack(L.w)
    y = B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS[act], residual=L.res)
    want, e = L.y64(act)
    T.assert_within(y, want, L.rounded(want, e), "y")
    # from the packed input: the values are the same, the order of the sums may not be
    z = torch.empty((M, N), dtype=L.type, device=Q.DEV)
    y2 = B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS[act], residual=L.res, x_packed=B.mx4_pack(L.x), z_out=z)
    T.assert_within(y2, want, L.rounded(want, e), "y of packed x")
    zw, ez = L.z64()
    T.assert_within(z, zw, L.rounded(zw, ez), "z")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("M,N,K", TILES)
def test_tiles(dtype, M, N, K):
    """Grids that fill the chip: tiles that end inside the matrix, from one block of columns to more than the ring holds."""
    L = Q.Layer(dtype, M, N, K, seed=K)
    w, z = B.mx4_pack(L.w), torch.empty((M, N), dtype=L.type, device=Q.DEV)
    y = B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS["gelu"], residual=L.res, z_out=z)
    want, e = L.y64("gelu")
    T.assert_within(y, want, L.rounded(want, e), "y")
    zw, ez = L.z64()
    T.assert_within(z, zw, L.rounded(zw, ez), "z")


@pytest.mark.parametrize("act", ["relu", "silu"])
@pytest.mark.parametrize("M,N,K", [(1, 48, 300), (40, 130, 300), (300, 520, 260)])
@pytest.mark.parametrize("bias,residual", [(False, False), (True, False), (False, True)])
def test_epilogue(act, M, N, K, bias, residual):
    L = Q.Layer("bf16", M, N, K, seed=7, bias=bias, residual=residual)
    y = B.mx4_linear(L.x, B.mx4_pack(L.w), N, bias=L.bias, act=T.ACTS[act], residual=L.res)
    want, e = L.y64(act)
    T.assert_within(y, want, L.rounded(want, e), "y")


@pytest.mark.parametrize("M,N,K", [(1, 50, 300), (7, 50, 301), (40, 131, 300), (300, 515, 260)])
def test_rows_apart_and_in_place(M, N, K):
    L = Q.Layer("fp16", M, N, K, seed=9)
    w = B.mx4_pack(L.w)
    plain = B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS["gelu"], residual=L.res)
    y, z = Q.apart(torch.zeros_like(plain), 5, 3), Q.apart(torch.zeros_like(plain))
    B.mx4_linear(Q.apart(L.x), w, N, bias=L.bias, act=T.ACTS["gelu"], residual=Q.apart(L.res), y_out=y, z_out=z)
    assert torch.equal(y, plain)
    assert (y._base.view(-1)[3:].view(M, N + 5)[:, N:] == 7).all() and (z._base.view(-1)[1:].view(M, N + 3)[:, N:] == 7).all()
    r = L.res.clone()
    B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS["gelu"], residual=r, y_out=r)
    assert torch.equal(r, plain)


@pytest.mark.parametrize("M,N,K", [(1, 64, 300), (9, 40, 300), (40, 130, 300), (300, 520, 260)])
def test_infinities_reach_their_own_outputs(M, N, K):
    L = Q.Layer("bf16", M, N, K, seed=11)
    w = B.mx4_pack(L.w)
    clean = B.mx4_linear(L.x, w, N, bias=L.bias)
    x = L.x.clone()
    x[M - 1, K - 1] = float("inf")
    y = B.mx4_linear(x, w, N, bias=L.bias)
    assert torch.isnan(y[M - 1]).all() and torch.equal(y[:M - 1], clean[:M - 1])
    bad = L.w.clone()
    bad[3, 0] = float("nan")
    y = B.mx4_linear(L.x, B.mx4_pack(bad), N, bias=L.bias)
    keep = [i for i in range(N) if i != 3]
    assert torch.isnan(y[:, 3]).all() and torch.equal(y[:, keep], clean[:, keep])


def test_far_scales():
    """Scales at the ends of the range: products that leave fp32 are infinite, those below it vanish, and a zero weight makes neither."""
    x = torch.zeros((1, 64), dtype=torch.bfloat16, device=Q.DEV)
    x[0, 0], x[0, 32] = 2.0 ** 100, 2.0 ** -100
    w = torch.zeros((4, 64), device=Q.DEV)
    w[0, 0], w[1, 0], w[2, 32], w[3, 32] = 2.0 ** 100, 2.0 ** -100, 2.0 ** -100, 2.0 ** 100
    for rows in (1, 40):
        y = B.mx4_linear(x.repeat(rows, 1), B.mx4_pack(w), 4)
        assert (y == torch.tensor([float("inf"), 1, 0, 1], device=Q.DEV)).all()


def test_same_arguments_same_bits_and_a_token_alone():
    L = Q.Layer("bf16", 40, 96, 700, seed=13)
    w = B.mx4_pack(L.w)
    first = B.mx4_linear(L.x, w, 96)
    assert all(torch.equal(first, B.mx4_linear(L.x, w, 96)) for _ in range(3))
    want, e = Q.Layer("bf16", 40, 96, 700, seed=13, bias=False, residual=False).y64("none")
    one = torch.cat([B.mx4_linear(L.x[i:i + 1], w, 96) for i in range(40)])
    T.assert_within(one, want, L.rounded(want, e), "one by one")
    assert B.mx4_linear(L.x[:0], w, 96).shape == (0, 96)


# ------------------------------------------------------------------ gradients

def grads64(L, act, seed, z):
    """dx, dw, dbias and bounds; z as the forward pass left it.  A dz within `slack` of the border of two codes, by the fp32 evaluation
    of the slope, may take either, which is a gap of its group: `moved` counts that in."""
    dy = Q.f64(L.dy)
    z64 = Q.f64(z) if z is not None else None
    s = T.slope(z64, act) if act != "none" else np.ones_like(dy)
    dz = dy * s
    slack = np.abs(dy) * (2.0 ** -21 * np.maximum(1, np.abs(z64))) if act in ("gelu", "silu") else np.zeros_like(dy)
    w, x = Q.f64(L.w), Q.f64(L.x)

    def either(d, sl, transposed):
        q = Q.four(d, seed, transposed)
        if not sl.any():
            return q, np.zeros_like(q)
        lo, hi = Q.four(d - sl, seed, transposed), Q.four(d + sl, seed, transposed)
        return q, np.maximum(np.abs(hi - q), np.abs(lo - q))

    q, mq = either(dz, slack, False)
    qt, mqt = either(dz.T, slack.T, True)
    wt, xt = Q.four(w.T), Q.four(x.T)
    dx, ex = q @ wt.T, mq @ np.abs(wt).T + (L.N + 2) * Q.EPS * ((np.abs(q) + mq) @ np.abs(wt).T) + L.N * 2.0 ** -126
    dw, ew = qt @ xt.T, mqt @ np.abs(xt).T + (L.M + 2) * Q.EPS * ((np.abs(qt) + mqt) @ np.abs(xt).T) + L.M * 2.0 ** -126
    return (dx, ex), (dw, ew), (dz.sum(0), slack.sum(0) + (L.M + 2) * Q.EPS * np.abs(dz).sum(0))


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("seed", [None, 77])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 40, 33), (31, 33, 70), (77, 130, 200), (260, 300, 130), (130, 600, 520)])
def test_backward(dtype, act, seed, M, N, K):
    L = Q.Layer(dtype, M, N, K, seed=M + N + K, residual=False)
    w, wt = B.mx4_pack(L.w, transposed=True)
    x, xt = B.mx4_pack(L.x, transposed=True)
    z = torch.empty((M, N), dtype=L.type, device=Q.DEV) if act != "none" else None
    B.mx4_linear(L.x, w, N, bias=L.bias, act=T.ACTS[act], x_packed=x, z_out=z)
    (dx, ex), (dw, ew), (db, eb) = grads64(L, act, seed, z)
    got = B.mx4_linear_backward(L.dy, wt, K, xt, act=T.ACTS[act], z=z, seed=Q.seed_tensor(seed), dw_dtype=torch.float32)
    T.assert_within(got[0], dx, L.rounded(dx, ex), "dx")
    T.assert_within(got[1], dw, ew, "dw")
    T.assert_within(got[2], db, L.rounded(db, eb), "dbias")
    assert got[1].dtype == torch.float32
    # rows apart; dw in 16 bits; and each output alone is the same as together
    r = B.mx4_linear_backward(Q.apart(L.dy), wt, K, xt, act=T.ACTS[act], z=None if z is None else Q.apart(z), seed=Q.seed_tensor(seed))
    assert torch.equal(r[0], got[0]) and torch.equal(r[2], got[2]) and torch.equal(r[1], got[1].to(L.type))
    for i in range(3):
        want = [i == k for k in range(3)]
        one = B.mx4_linear_backward(L.dy, wt, K, xt, act=T.ACTS[act], z=z, seed=Q.seed_tensor(seed), want_dx=want[0], want_dw=want[1],
                                    want_dbias=want[2], dw_dtype=torch.float32)
        assert torch.equal(one[i], got[i]) and all(one[k] is None for k in range(3) if k != i)


@pytest.mark.parametrize("act", ["none", "relu"])
def test_backward_against_differences(act):
    """Where all values are codes under both groupings the layer is its plain form, and a difference is exact: a step of x or w by
    one of those values, on integers that fp32 and bfloat16 sum exactly."""
    rng = np.random.default_rng(21)
    M, N, K = 40, 36, 34
    pick = lambda *shape: rng.choice([-4.0, -3.0, -2.0, -1.0, 0.0, 1.0, 2.0, 3.0, 4.0], shape)
    x, w, dy = pick(M, K), pick(N, K), rng.choice([-1.0, 0.0, 1.0, 4.0], (M, N))
    x[::8], x[:, ::8], w[::8], w[:, ::8], dy[::8], dy[:, ::8] = 4, 4, 4, 4, 4, 4    # every group's scale is 1
    dev = lambda v: torch.from_numpy(v.astype(np.float32)).to(Q.DEV)
    X, DY = dev(x).bfloat16(), dev(dy).bfloat16()
    wp, wt = B.mx4_pack(dev(w), transposed=True)
    _, xt = B.mx4_pack(X, transposed=True)
    z = torch.empty((M, N), dtype=torch.float16, device=Q.DEV)
    y = B.mx4_linear(X.half(), wp, N, act=T.ACTS[act], z_out=z)                   # |z| <= 16 * 34 = 544: exact in float16
    Q.equal(y, T.act(x @ w.T, act))
    dx, dw, _ = B.mx4_linear_backward(DY.half(), wt, K, xt, act=T.ACTS[act], z=z if act != "none" else None, dw_dtype=torch.float32)
    loss = lambda x, w: (dy * T.act(x @ w.T, act)).sum()
    h = 2.0 ** -20                                                                # no z crosses 0 but those that are 0
    z0 = x @ w.T
    for _ in range(40):
        m, n, k = rng.integers(M), rng.integers(N), rng.integers(K)
        for arr, idx, got in ((x, (m, k), dx), (w, (n, k), dw)):
            up, down = arr.copy(), arr.copy()
            up[idx] += h
            down[idx] -= h
            pair = ((up, w), (down, w)) if arr is x else ((x, up), (x, down))
            if act == "relu" and (z0[m] == 0).any() or act == "relu" and (z0[:, n] == 0).any():
                continue
            diff = (loss(*pair[0]) - loss(*pair[1])) / (2 * h)
            assert abs(float(got[idx]) - diff) <= 2.0 ** -11 * abs(diff) + 1e-6, (idx, float(got[idx]), diff)


def test_backward_of_no_tokens():
    w, wt = B.mx4_pack(torch.randn((50, 40), device=Q.DEV), transposed=True)
    dy = torch.empty((0, 50), dtype=torch.bfloat16, device=Q.DEV)
    none = torch.empty(0, dtype=torch.uint8, device=Q.DEV)
    dx, dw, db = B.mx4_linear_backward(dy, wt, 40, none, dw=torch.full((50, 40), 3.0, device=Q.DEV), dbias=torch.full((50,), 3.0, device=Q.DEV).bfloat16())
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("seed", [None, 5])
@pytest.mark.parametrize("M,N,K", [(3, 40, 33), (130, 200, 70)])
def test_gradient_behind_a_relu_that_is_off(dtype, seed, M, N, K):
    """An infinity or NaN in dy where the relu is off reaches nothing, as zeros there; where it is on it reaches its token and its output."""
    L = Q.Layer(dtype, M, N, K, seed=M, residual=False)
    wt, xt = B.mx4_pack(L.w, transposed=True)[1], B.mx4_pack(L.x, transposed=True)[1]
    z = Q.values(np.random.default_rng(7), M, N, dtype)
    kw = dict(act=B.RTN_ACT_RELU, z=z, seed=Q.seed_tensor(seed), dw_dtype=torch.float32)
    z[M // 2, N // 2] = z[0, 0] = -1.0
    z[M - 1, N - 1] = 0.0
    want = B.mx4_linear_backward(L.dy, wt, K, xt, **kw)
    dy = L.dy.clone()
    dy[M // 2, N // 2], dy[0, 0], dy[M - 1, N - 1] = float("inf"), float("nan"), float("-inf")
    for a, b in zip(B.mx4_linear_backward(dy, wt, K, xt, **kw), want):
        assert torch.equal(a, b)
    z[M // 2, N // 2] = 1.0
    want = B.mx4_linear_backward(L.dy, wt, K, xt, **kw)
    dx, dw, db = B.mx4_linear_backward(dy, wt, K, xt, **kw)
    rows, cols = torch.arange(M, device=Q.DEV) != M // 2, torch.arange(N, device=Q.DEV) != N // 2
    assert torch.isnan(dx[M // 2]).all() and torch.equal(dx[rows], want[0][rows])
    assert torch.isnan(dw[N // 2]).all() and torch.equal(dw[cols], want[1][cols])
    assert not torch.isfinite(db[N // 2]) and torch.equal(db[cols], want[2][cols])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["gelu", "silu"])
@pytest.mark.parametrize("M,N,K", [(3, 40, 33), (130, 200, 70)])
def test_slopes_far_out(dtype, act, M, N, K):
    """z at the ends of its type, to which float16 rounds what is beyond them: the slopes are 1 and 0, as a relu's; a NaN stays one."""
    L = Q.Layer(dtype, M, N, K, seed=M, residual=False)
    wt, xt = B.mx4_pack(L.w, transposed=True)[1], B.mx4_pack(L.x, transposed=True)[1]
    sign = torch.from_numpy(np.random.default_rng(8).choice([-1.0, 1.0], (M, N)).astype(np.float32)).to(Q.DEV).to(L.type)
    for seed in (None, 6):
        kw = dict(seed=Q.seed_tensor(seed), dw_dtype=torch.float32)
        want = B.mx4_linear_backward(L.dy, wt, K, xt, act=B.RTN_ACT_RELU, z=sign, **kw)
        for far in (float("inf"), float(torch.finfo(L.type).max), 200.0):
            for a, b in zip(B.mx4_linear_backward(L.dy, wt, K, xt, act=T.ACTS[act], z=sign * far, **kw), want):
                assert torch.equal(a, b), far
    z = sign * float("inf")
    z[1, 2] = float("nan")
    dx, dw, db = B.mx4_linear_backward(L.dy, wt, K, xt, act=T.ACTS[act], z=z, dw_dtype=torch.float32)
    assert torch.isnan(dx[1]).all() and torch.isnan(dw[2]).all() and torch.isnan(db[2])
    assert torch.isfinite(dx[0]).all() and torch.isfinite(dw[0]).all()


# ------------------------------------------------------------------ streams, graphs, buffers

def test_captured_step_takes_new_inputs_and_seeds():
    """A training step and a token's answer in a graph, replayed with other inputs and another seed between eager work, against eager
    calls."""
    M, N, K = 70, 130, 200
    L = [Q.Layer("bf16", M, N, K, seed=s) for s in (1, 2, 3)]
    hold = dict(x=L[0].x.clone(), dy=L[0].dy.clone(), w=L[0].w.clone(), seed=Q.seed_tensor(5))

    def step(x, dy, w, seed):
        wp, wt = B.mx4_pack(w, transposed=True)
        xp, xt = B.mx4_pack(x, transposed=True)
        z = torch.empty((M, N), dtype=x.dtype, device=x.device)
        y = B.mx4_linear(x, wp, N, act=T.ACTS["relu"], x_packed=xp, z_out=z)
        one = B.mx4_linear(x[:1], wp, N)
        many = B.mx4_linear(x, wp, N)
        return (y, one, many) + tuple(B.mx4_linear_backward(dy, wt, K, xt, act=T.ACTS["relu"], z=z, seed=seed))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(**hold)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(**hold)
    for i in (1, 2, 0, 1):
        for k in ("x", "dy", "w"):
            hold[k].copy_(getattr(L[i], k))
        hold["seed"].fill_(100 + i)
        graph.replay()
        eager = step(L[i].x, L[i].dy, L[i].w, Q.seed_tensor(100 + i))
        torch.cuda.synchronize()
        for a, b in zip(out, eager):
            assert torch.equal(a, b)


def test_two_streams_at_once():
    L = [Q.Layer("fp16", 60, 200, 300, seed=s) for s in (1, 2)]
    packed = [B.mx4_pack(l.w, transposed=True) for l in L]

    def work(l, p):
        _, xt = B.mx4_pack(l.x, transposed=True)
        return (B.mx4_linear(l.x, p[0], 200),) + tuple(B.mx4_linear_backward(l.dy, p[1], 300, xt))

    want = [work(l, p) for l, p in zip(L, packed)]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(work(L[i], packed[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for g in got[i] for a, b in zip(g, want[i]))


def test_buffers():
    L = Q.Layer("bf16", 40, 64, 96, seed=3)
    w, wt = B.mx4_pack(L.w, transposed=True)
    _, xt = B.mx4_pack(L.x, transposed=True)
    for call, size in ((lambda ws: B.mx4_linear(L.x, w, 64, workspace=ws), B.lib().rtn_mx4_linear_workspace_bytes(40, 64, 96)),
                       (lambda ws: B.mx4_linear_backward(L.dy, wt, 96, xt, workspace=ws), B.lib().rtn_mx4_linear_backward_workspace_bytes(40, 64, 96))):
        assert size > 0
        for bad in (torch.empty(size, dtype=torch.uint8), torch.empty(2 * size, dtype=torch.uint8, device=Q.DEV)[::2]):
            with pytest.raises(ValueError):
                call(bad)
        with pytest.raises(B.RtnError) as e:
            call(torch.empty(size - 1, dtype=torch.uint8, device=Q.DEV))
        assert e.value.status == B.RTN_ERR_WORKSPACE
    with pytest.raises(ValueError):
        B.mx4_linear(L.x, w[:-1], 64)
    with pytest.raises(ValueError):
        B.mx4_linear_backward(L.dy, wt, 96, xt[:-1])
    with pytest.raises(AssertionError):
        B.mx4_linear(L.x.float(), w, 64)
    with pytest.raises(AssertionError):
        B.mx4_linear(L.x, w, 64, residual=L.res[:-1])
    with pytest.raises(AssertionError):
        B.mx4_pack(L.x.t())
    with pytest.raises(AssertionError):
        B.mx4_pack(L.x, seed=torch.zeros(2, dtype=torch.int64, device=Q.DEV))
    with pytest.raises(AssertionError):
        B.mx4_unpack(w, 64, 96, torch.float64)
    with pytest.raises(B.RtnError):
        B.mx4_linear(L.x, w, 64, act=9)
    with pytest.raises(B.RtnError) as e:
        B.mx4_linear_backward(L.dy, wt, 96, xt, act=B.RTN_ACT_RELU)
    assert e.value.status == B.RTN_ERR_NULL


# ------------------------------------------------------------------ every form of the product

@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("act", ["none", "silu"])
@pytest.mark.parametrize("M,N,K", [s for s in SIZES if s[0] <= 16])
def test_z_of_a_few_tokens(dtype, act, M, N, K):
    """The value before the activation where the tokens are packed on the way."""
    L = Q.Layer(dtype, M, N, K, seed=M + N + K + 1)
    z = torch.empty((M, N), dtype=L.type, device=Q.DEV)
    B.mx4_linear(L.x, B.mx4_pack(L.w), N, bias=L.bias, act=T.ACTS[act], residual=L.res, z_out=z)
    want, e = L.z64()
    T.assert_within(z, want, L.rounded(want, e), "z")


# The larger forms, one size each, and one whose residual is read past the caches: edges of tiles inside, whole ones beside them
FORMS = [(1300, 1290, 200), (1797, 1750, 330), (3001, 2990, 140), (4200, 4100, 140), (4200, 8200, 140)]


def _product64(L):
    """Q(x) Q(w)^T in 64 bits and the sums of its terms' magnitudes."""
    x, w = Q.four(Q.f64(L.x)), Q.four(Q.f64(L.w))
    return x @ w.T, np.abs(x) @ np.abs(w).T


@pytest.mark.parametrize("dtype,M,N,K", [(("bf16", "fp16")[i % 2],) + s for i, s in enumerate(FORMS)])
def test_epilogue_of_every_form(dtype, M, N, K):
    L = Q.Layer(dtype, M, N, K, seed=K + N)
    w, (s, size) = B.mx4_pack(L.w), _product64(L)
    for act, bias, residual in (("none", False, False), ("relu", False, True), ("silu", True, False), ("none", True, True)):
        b = Q.f64(L.bias) if bias else np.zeros(N)
        z, ez = s + b, (K + 2) * Q.EPS * (size + np.abs(b)) + K * 2.0 ** -126
        want, e = T.act(z, act), 1.13 * ez + (Q.ACT_EPS * np.maximum(1, np.abs(z)) if act == "silu" else 0)
        if residual:
            r = Q.f64(L.res)
            want, e = want + r, e + Q.EPS * (np.abs(want + r) + np.abs(r))
        y = B.mx4_linear(L.x, w, N, bias=L.bias if bias else None, act=T.ACTS[act], residual=L.res if residual else None)
        T.assert_within(y, want, L.rounded(want, e), "y, %s" % act)


@pytest.mark.parametrize("M,N,K", FORMS)
def test_rows_apart_in_place_and_infinities_of_every_form(M, N, K):
    """Against the same call on dense rows and buffers of its own, to the bit."""
    L = Q.Layer("bf16", M, N, K, seed=K)
    w, kw = B.mx4_pack(L.w), dict(bias=L.bias, act=T.ACTS["silu"])
    z = torch.empty((M, N), dtype=L.type, device=Q.DEV)
    plain = B.mx4_linear(L.x, w, N, residual=L.res, z_out=z, **kw)
    ya, za = Q.apart(torch.zeros_like(plain), 5, 3), Q.apart(torch.zeros_like(plain))
    B.mx4_linear(Q.apart(L.x), w, N, residual=Q.apart(L.res, 7, 5), y_out=ya, z_out=za, **kw)
    assert torch.equal(ya, plain) and torch.equal(za, z)
    assert (ya._base.view(-1)[3:].view(M, N + 5)[:, N:] == 7).all() and (za._base.view(-1)[1:].view(M, N + 3)[:, N:] == 7).all()
    r = L.res.clone()
    B.mx4_linear(L.x, w, N, residual=r, y_out=r, **kw)
    assert torch.equal(r, plain)
    r = Q.apart(L.res, 3, 1)
    B.mx4_linear(L.x, w, N, residual=r, y_out=r, **kw)
    assert torch.equal(r, plain) and (r._base.view(-1)[1:].view(M, N + 3)[:, N:] == 7).all()
    x = L.x.clone()
    x[M - 1, K - 1] = float("inf")
    y = B.mx4_linear(x, w, N, residual=L.res, **kw)
    assert torch.isnan(y[M - 1]).all() and torch.equal(y[:M - 1], plain[:M - 1])
    bad = L.w.clone()
    bad[3, 0] = float("nan")
    y = B.mx4_linear(L.x, B.mx4_pack(bad), N, residual=L.res, **kw)
    keep = torch.arange(N, device=Q.DEV) != 3
    assert torch.isnan(y[:, 3]).all() and torch.equal(y[:, keep], plain[:, keep])


# (M, N, K) whose dx, a product of M x K over N, or dw, of N x K over M, takes one of those forms; a multiple of every tile among them, and
# more blocks of 128 to contract over than the rings hold
GRADS = [(200, 1300, 1290), (1300, 200, 1290), (260, 1800, 1750), (1800, 700, 1750), (130, 3001, 2990), (3001, 130, 2990), (700, 2900, 3001),
         (96, 3328, 3328), (300, 4200, 4100), (4200, 70, 4100)]


@pytest.mark.parametrize("dtype,act,seed,M,N,K", [(("bf16", "fp16")[i % 2], ("none", "relu")[i // 2 % 2], (77, None, 78)[i % 3]) + s for i, s in enumerate(GRADS)])
def test_gradients_of_every_form(dtype, act, seed, M, N, K):
    L = Q.Layer(dtype, M, N, K, seed=M + N, residual=False)
    wt, xt = B.mx4_pack(L.w, transposed=True)[1], B.mx4_pack(L.x, transposed=True)[1]
    z = Q.values(np.random.default_rng(N), M, N, dtype) if act != "none" else None
    kw = dict(act=T.ACTS[act], z=z, seed=Q.seed_tensor(seed))
    (dx, ex), (dw, ew), (db, eb) = grads64(L, act, seed, z)
    got = B.mx4_linear_backward(L.dy, wt, K, xt, dw_dtype=torch.float32, **kw)
    T.assert_within(got[0], dx, L.rounded(dx, ex), "dx")
    T.assert_within(got[1], dw, ew, "dw")
    T.assert_within(got[2], db, L.rounded(db, eb), "dbias")
    out = Q.apart(torch.zeros_like(got[0]), 5, 3)
    r = B.mx4_linear_backward(Q.apart(L.dy), wt, K, xt, dx=out, **kw)
    assert torch.equal(out, got[0]) and torch.equal(r[1], got[1].to(L.type)) and torch.equal(r[2], got[2])
    assert (out._base.view(-1)[3:].view(M, K + 5)[:, K:] == 7).all()
