"""The ternary linear layer, its 8-bit activation checkpoints and its gradients against plain 64-bit forms."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu

# one token, a few, the edges of the kernels' token counts and tiles (32, 64, 128, 256), odd sizes, rows that are no whole
# 16 bytes, columns that end inside a 64-step, and enough tiles for each tile size
SIZES = [(1, 64, 64), (1, 4096, 1024), (2, 33, 70), (7, 100, 1000), (31, 250, 264), (32, 96, 2187), (33, 256, 256), (64, 65, 1),
         (65, 1, 130), (100, 31, 63), (129, 300, 200), (257, 515, 1027), (700, 1100, 328), (1800, 1800, 72), (3700, 3700, 40),
         (9, 4160, 520), (16, 100, 520), (300, 900, 1000), (500, 1500, 2187), (1100, 1000, 2000)]


def run(L, name, w, **kw):
    return B.linear(L.x, w, L.N, L.alpha, bias=L.bias, act=T.ACTS[name], residual=L.res, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", SIZES)
def test_forward(dtype, size):
    M, N, K = size
    print("[case] linear forward", dtype, size, flush=True)
    acts = ["none", "relu", "gelu", "silu"] if M * N <= 1 << 18 else [["none", "relu", "gelu", "silu"][(M + N + K) % 4]]
    L = T.Layer(dtype, M, N, K, seed=M + 7 * N + 31 * K)
    w = B.linear_prepare(L.codes, N, K)
    for name in acts:
        y, e = L.y64(name)
        T.assert_within(run(L, name, w), y, L.rounded(y, e), "y, %s" % name)
        z8 = B.checkpoint_empty(M, N, T.DEV)
        T.assert_within(run(L, name, w, z_ckpt=z8), y, L.rounded(y, e), "y with a checkpoint, %s" % name)
        z, ez = L.z64()
        zhat, scale = T.eight_bits(z, dtype)
        # half a step, or a whole one of the next scale where the group's maximum lies on the border between two
        T.assert_within(B.checkpoint_unpack(z8, M, N, L.type), z, scale * (1 + 1e-9) + 2 * ez, "z^")
        near = T.f64(B.checkpoint_unpack(z8, M, N, L.type)) == zhat
        assert near.mean() > 0.98, near.mean()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", SIZES)
def test_backward(dtype, size):
    M, N, K = size
    print("[case] linear backward", dtype, size, flush=True)
    acts = ["none", "relu", "gelu", "silu"] if M * max(N, K) <= 1 << 18 else [["gelu", "silu", "relu", "none"][(M + N + K) % 4]]
    L = T.Layer(dtype, M, N, K, seed=M + 5 * N + 3 * K, vector=(M + N) % 3 != 0)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    x8 = B.checkpoint_pack(L.x)
    xhat = T.f64(B.checkpoint_unpack(x8, M, K, L.type))
    assert (xhat == T.eight_bits(T.f64(L.x), dtype)[0]).all()
    for name in acts:
        z8 = None
        zhat = np.zeros((M, N))
        if name != "none":
            z8 = B.checkpoint_empty(M, N, T.DEV)
            run(L, name, w, z_ckpt=z8)
            zhat = T.f64(B.checkpoint_unpack(z8, M, N, L.type))
        (dx, ex), (dw, ew), (db, eb) = L.grads64(name, xhat, zhat)
        got = B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS[name], z_ckpt=z8)
        T.assert_within(got[0], dx, L.rounded(dx, ex), "dx, %s" % name)
        T.assert_within(got[1], dw, L.rounded(dw, ew), "dw, %s" % name)
        T.assert_within(got[2], db, L.rounded(db, eb), "dbias, %s" % name)
        # one at a time, dw in 32 bits
        f32 = B.linear_backward(L.dy, None, K, L.alpha, x8, act=T.ACTS[name], z_ckpt=z8, want_dx=False, want_dbias=False, dw_dtype=torch.float32)
        assert f32[0] is None and f32[2] is None
        T.assert_within(f32[1], dw, ew, "dw in fp32, %s" % name)
        only = B.linear_backward(L.dy, wt, K, L.alpha, None, act=T.ACTS[name], z_ckpt=z8, want_dw=False, want_dbias=False)
        assert torch.equal(only[0], got[0])
        only = B.linear_backward(L.dy, None, K, L.alpha, None, act=T.ACTS[name], z_ckpt=z8, want_dx=False, want_dw=False)
        assert torch.equal(only[2], got[2])


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", [(1, 1), (1, 64), (31, 7), (32, 128), (33, 129), (100, 1000), (1000, 136), (77, 2187)])
def test_checkpoint(dtype, size):
    """Bit for bit what the definition says, with the values where it can go wrong among the inputs."""
    M, C = size
    print("[case] checkpoint", dtype, size, flush=True)
    rng = np.random.default_rng(M * C)
    v = rng.standard_normal((M, C)) * np.exp2(rng.integers(-12, 12, C))
    v[:, rng.random(C) < 0.1] = 0
    v[:, rng.random(C) < 0.1] *= 2.0 ** -12          # float16: into its subnormal values
    tiny, big = (2.0 ** -133, 3.3895313892515355e38) if dtype == "bf16" else (2.0 ** -24, 65504.0)
    specials = [127.0, -127.5, 127.75 if dtype == "fp16" else 127.0, 128.0, 63.5, 64.0, tiny, -tiny, big, -big, 0.0, -0.0, 3 * tiny, 126.5 * tiny]
    for i, s in enumerate(specials):
        c = i % C
        v[rng.integers(0, M), c] = s
    x = torch.from_numpy(v).to(T.TYPES[dtype]).to(T.DEV)
    assert torch.isfinite(x).all()
    ckpt = B.checkpoint_pack(x)
    back = B.checkpoint_unpack(ckpt, M, C, T.TYPES[dtype])
    want, scale = T.eight_bits(T.f64(x), dtype)
    assert np.array_equal(T.f64(back), want)
    assert np.isfinite(want).all()
    end = np.abs(T.f64(x)) > 127.5 * scale                  # the end of the type's range
    assert (np.abs(T.f64(x) - want) <= np.where(end, scale, scale / 2)).all()
    # a group with an infinity or NaN reads back as NaN, the others as before
    if M > 1 and C > 4:
        x[0, 1], x[M - 1, 3] = float("inf"), float("nan")
        want = T.eight_bits(T.f64(x), dtype)[0]
        assert np.array_equal(T.f64(B.checkpoint_unpack(B.checkpoint_pack(x), M, C, T.TYPES[dtype])), want, equal_nan=True)


def test_gradients_against_differences():
    """Inputs and weights whose checkpoints are exact (x whole numbers up to 15, z multiples of 1/16 below 7.5 in magnitude): the
    gradients against central differences of the 64-bit loss sum(dy * y).  A difference of step h = 2^-10 is off by h^2 / 6
    times the third derivative along its direction (below 2 per unit), a thousandth of u."""
    for dtype in ("bf16", "fp16"):
        for name in ("none", "gelu", "silu"):
            M, N, K = 40, 24, 8
            L = T.Layer(dtype, M, N, K, seed=11, bias=False, residual=False, vector=False)
            rng = np.random.default_rng(12)
            xv = rng.integers(-15, 16, (M, K)).astype(np.float64)
            L.x, L.alpha = torch.from_numpy(xv).to(L.type).to(T.DEV), 1.0 / 16
            w, wt = B.linear_prepare(L.codes, N, K, backward=True)
            z8 = B.checkpoint_empty(M, N, T.DEV)
            B.linear(L.x, w, N, L.alpha, act=T.ACTS[name], z_ckpt=z8)
            x8, dy = B.checkpoint_pack(L.x), T.f64(L.dy)
            wv = L.t / 16.0
            loss = lambda x, ww: float((dy * T.act(x @ ww.T, name)).sum())
            got = B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS[name], z_ckpt=z8, dw_dtype=torch.float32)
            (dx, ex), (dw, ew), _ = L.grads64(name, xv, xv @ wv.T)
            h = 2.0 ** -10
            for g, at, e in ((got[0], "x", L.rounded(dx, ex)), (got[1], "w", ew)):
                for _ in range(24):
                    i = tuple(rng.integers(0, s) for s in g.shape)
                    d = np.zeros(g.shape)
                    d[i] = h
                    diff = (loss(xv + d, wv) - loss(xv - d, wv) if at == "x" else loss(xv, wv + d) - loss(xv, wv - d)) / (2 * h)
                    third = (np.abs(dy).sum() * (15 if at == "w" else 1) ** 3) * h * h
                    assert abs(float(g[i]) - diff) <= e[i] + third + 1e-9 * abs(diff), (dtype, name, at, i, float(g[i]), diff, e[i], third)


def test_formats_prepare_alike():
    rng = np.random.default_rng(3)
    for N, K in ((1, 1), (33, 70), (130, 515)):
        t = rng.integers(-1, 2, (N, K))
        bufs = [B.linear_prepare(T.codes_of(t, f), N, K, fmt=f, backward=True) for f in (B.RTN_CODE_I8, B.RTN_CODE_FP4, B.RTN_CODE_BITPLANE)]
        for w, wt in bufs[1:]:
            assert torch.equal(w, bufs[0][0]) and torch.equal(wt, bufs[0][1])
        assert torch.equal(B.linear_prepare(T.codes_of(np.ascontiguousarray(t.T)), K, N), bufs[0][1])


@pytest.mark.parametrize("size", [(3, 70, 200), (40, 70, 200), (300, 136, 264)])
def test_strides_alignment_and_places(size):
    """Rows that lie apart, views that start inside 16 bytes, y in the residual's place: the same bits as dense tensors."""
    M, N, K = size
    print("[case] strides", size, flush=True)
    for dtype in ("bf16", "fp16"):
        L = T.Layer(dtype, M, N, K, seed=M)
        w, wt = B.linear_prepare(L.codes, N, K, backward=True)
        z = B.checkpoint_empty(M, N, T.DEV)
        y = run(L, "gelu", w, z_ckpt=z)
        x8 = B.checkpoint_pack(L.x)
        grads = B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS["gelu"], z_ckpt=z)

        def apart(t, pad, start):
            buf = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device=T.DEV)
            v = buf[:, start:start + t.shape[1]]
            v.copy_(t)
            return v
        for pad, start in ((8, 0), (8, 8), (5, 0), (3, 1)):
            x, r, dy = (apart(t, pad, start) for t in (L.x, L.res, L.dy))
            out = apart(torch.zeros_like(L.dy), pad, start)
            base = out._base if out._base is not None else out
            z2 = B.checkpoint_empty(M, N, T.DEV)
            B.linear(x, w, N, L.alpha, bias=L.bias, act=T.ACTS["gelu"], residual=r, y_out=out, z_ckpt=z2)
            assert torch.equal(out, y)
            assert torch.isnan(base).sum().item() == M * pad          # nothing is written between the rows
            assert torch.equal(B.checkpoint_unpack(z2, M, N, L.type), B.checkpoint_unpack(z, M, N, L.type))
            B.linear(x, w, N, L.alpha, bias=L.bias, act=T.ACTS["gelu"], residual=r, y_out=r)
            ref = run(L, "gelu", w)
            assert torch.equal(r, ref)
            x8b = B.checkpoint_pack(x)
            assert torch.equal(B.checkpoint_unpack(x8b, M, K, L.type), B.checkpoint_unpack(x8, M, K, L.type))
            back = apart(torch.zeros_like(L.x), pad, start)
            B.checkpoint_unpack(x8b, M, K, L.type, out=back)
            assert torch.equal(back, B.checkpoint_unpack(x8, M, K, L.type))
            dx = apart(torch.zeros_like(L.x), pad, start)
            g = B.linear_backward(dy, wt, K, L.alpha, x8b, act=T.ACTS["gelu"], z_ckpt=z2, dx=dx)
            assert all(torch.equal(a, b) for a, b in zip(g, grads))
            s = 1.25
            a = B.linear_backward(dy, wt, K, s, x8b)
            b = B.linear_backward(L.dy, wt, K, s, x8)
            assert all(torch.equal(p, q) for p, q in zip(a, b))


def test_no_tokens():
    L = T.Layer("bf16", 4, 70, 100, seed=1)
    w, wt = B.linear_prepare(L.codes, 70, 100, backward=True)
    x, dy = L.x[:0], L.dy[:0]
    x8, z8 = B.checkpoint_pack(x), B.checkpoint_empty(0, 70, T.DEV)
    assert B.checkpoint_unpack(x8, 0, 100, L.type).shape == (0, 100)
    assert B.linear(x, w, 70, L.alpha, bias=L.bias, z_ckpt=z8).shape == (0, 70)
    dx, dw, db = B.linear_backward(dy, wt, 100, L.alpha, x8, act=T.ACTS["gelu"], z_ckpt=z8,
                                   dw=torch.full((70, 100), 7.0, dtype=L.type, device=T.DEV), dbias=torch.full((70,), 7.0, dtype=L.type, device=T.DEV))
    assert dx.shape == (0, 100) and not dw.any() and not db.any()


@pytest.mark.parametrize("M", [5, 70])
def test_infinities_and_nans_stay_in_their_rows(M):
    for name in ("none", "relu", "gelu", "silu"):
        L = T.Layer("bf16", M, 48, 136, seed=2)
        w, wt = B.linear_prepare(L.codes, 48, 136, backward=True)
        clean = run(L, name, w)
        L.x[1, 5] = float("nan")
        L.x[3, 7] = float("inf")
        y = run(L, name, w)
        keep = [m for m in range(M) if m not in (1, 3)]
        assert torch.equal(y[keep], clean[keep])
        assert torch.isnan(y[1]).all()
        t7 = L.t[:, 7]                                       # 0 * inf is a NaN, as in any product
        got = T.f64(y[3])
        assert np.isnan(got[t7 == 0]).all() and not np.isfinite(got[t7 > 0]).any()
        # the group of 32 tokens of the poisoned channels gives NaN gradients, the other channels and groups do not
        x8 = B.checkpoint_pack(L.x)
        dw = T.f64(B.linear_backward(L.dy, wt, 136, L.alpha, x8, want_dx=False, want_dbias=False)[1])
        bad = np.isnan(dw).all(axis=0)
        assert bad[5] and bad[7] and bad.sum() == 2 and not np.isnan(dw[:, ~bad]).any()


def test_zero_weights_and_rows():
    """Weights that are all zero leave bias and residual; a group of zeros is kept as zeros."""
    L = T.Layer("fp16", 50, 40, 72, seed=5, zeros=1.1)
    w, wt = B.linear_prepare(L.codes, 40, 72, backward=True)
    y, e = L.y64("none")
    T.assert_within(run(L, "none", w), y, L.rounded(y, e), "y")
    x8 = B.checkpoint_pack(torch.zeros_like(L.x))
    dx, dw, db = B.linear_backward(L.dy, wt, 72, L.alpha, x8)
    assert not dx.any() and not dw.any() and db.any()


def test_same_bits_twice_and_on_another_stream():
    for M, N, K in ((3, 4096, 1024), (500, 600, 264)):
        L = T.Layer("bf16", M, N, K, seed=9)

        def step():
            w, wt = B.linear_prepare(L.codes, N, K, backward=True)
            x8, z8 = B.checkpoint_pack(L.x), B.checkpoint_empty(M, N, T.DEV)
            y = run(L, "silu", w, z_ckpt=z8)
            return (y,) + B.linear_backward(L.dy, wt, K, L.alpha, x8, act=T.ACTS["silu"], z_ckpt=z8)
        first = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, step()))
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            other = step()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(first, other))


def test_recorded_in_a_graph():
    """A serving step and a training step replayed from a graph, against the eager calls, with other work in between."""
    M, N, K = 4, 512, 256
    L, L2 = T.Layer("bf16", M, N, K, seed=1), T.Layer("bf16", 96, N, K, seed=2)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    y, x, dy = torch.empty(M, N, dtype=L.type, device=T.DEV), L.x.clone(), L2.dy.clone()
    x8, ws = B.checkpoint_pack(L2.x), torch.empty(B.lib().rtn_linear_backward_workspace_bytes(96, N, K), dtype=torch.uint8, device=T.DEV)
    dx, dw, db = B.linear_backward(dy, wt, K, L.alpha, x8, workspace=ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        B.linear(x, w, N, L.alpha, bias=L.bias, y_out=y)
        B.linear_backward(dy, wt, K, L.alpha, x8, dx=dx, dw=dw, dbias=db, workspace=ws)
    for i in range(4):
        x.copy_(L.x * (i + 1))
        dy.copy_(L2.dy.roll(i, 0))
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, B.linear(x, w, N, L.alpha, bias=L.bias))
        want = B.linear_backward(dy, wt, K, L.alpha, x8)
        assert all(torch.equal(a, b) for a, b in zip((dx, dw, db), want))


def test_offsets_beyond_32_bits():
    """A tensor of more than 2^31 elements (4.6 GB): its last rows against the same rows by themselves."""
    M, N, K = 70016, 64, 32768
    print("[case] linear, 70016 x 32768", flush=True)
    rng = np.random.default_rng(4)
    t = rng.integers(-1, 2, (N, K))
    w, wt = B.linear_prepare(T.codes_of(t), N, K, backward=True)
    x = torch.zeros((M, K), dtype=torch.bfloat16, device=T.DEV)
    part = torch.randn((96, K), device=T.DEV).to(torch.bfloat16)
    x[-96:] = part
    y = B.linear(x, w, N, 0.01, act=B.RTN_ACT_SILU)
    P = T.Layer("bf16", 96, N, K, seed=5, bias=False, residual=False, vector=False)
    P.x, P.alpha, P.t = part, 0.01, t
    want, e = P.y64("silu")
    T.assert_within(y[-96:], want, P.rounded(want, e), "y")
    assert not y[:-96].any()
    x8 = B.checkpoint_pack(x)
    back = B.checkpoint_unpack(x8, M, K, torch.bfloat16)
    assert torch.equal(back[-96:], B.checkpoint_unpack(B.checkpoint_pack(part), 96, K, torch.bfloat16))
    dy = torch.randn((M, N), device=T.DEV).to(torch.bfloat16)
    dx, dw, db = B.linear_backward(dy, wt, K, 0.01, x8, dw_dtype=torch.float32)
    L = T.Layer("bf16", 96, N, K, seed=6)
    L.dy, L.alpha, L.t = dy[-96:].contiguous(), 0.01, t
    (dxs, ex), (dws, ew), _ = L.grads64("none", T.f64(back[-96:]), None)
    T.assert_within(dx[-96:], dxs, L.rounded(dxs, ex), "dx")
    T.assert_within(dw, dws, ew, "dw")                       # only the last rows of x are not zero


def test_feed_forward_block_trains_and_answers():
    """The example: the loss against a teacher falls, and one token alone is answered as among others (the forms add in other
    orders, and h is rounded to 16 bits in between: two roundings of y and one of h of an ulp each)."""
    from paper_1912_02057_amd import ternary_mlp as E
    block, losses = E.train(steps=40, tokens=256, width=128, hidden=320)
    assert losses[-1] < 0.75 * losses[0], losses
    block.freeze()
    x = torch.randn((40, 128), device=T.DEV).to(torch.bfloat16)
    y, one = T.f64(block(x)), np.concatenate([T.f64(block(x[i:i + 1])) for i in range(40)])
    h = T.f64(block.up(x, T.ACTS["gelu"]))
    t2 = np.abs(T.f64(block.down.w)) > E.THRESHOLD
    bound = 2 * T.U["bf16"] * np.maximum(np.abs(y), np.abs(one)) + 2 * T.U["bf16"] * (np.abs(h) @ t2.T) * T.f64(block.down.alpha)
    T.assert_within(one, y, bound, "one token")
