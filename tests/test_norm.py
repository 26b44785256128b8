"""Norms around a block and their gradients against their formulas in 64 bits.

Bounds, eps = 2^-24 that of fp32, u that of the 16-bit type.  The sum of C squares is off by at most (C + 1) eps of itself, so 1 / sqrt(mean + e) by
half of that and a few roundings: R = (C / 2 + 8) eps.  The mean of a row is off by C eps mean |v|, which n takes on as that times r.
What follows is a handful of fp32 operations on each value, each off by eps of its operands' size, and one rounding to 16 bits."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T
import mx4_testlib as Q
from mx4_testlib import collected  # noqa: F401 (a fixture of the module)

pytestmark = pytest.mark.gpu

EPS = Q.EPS
KINDS = {"rms": B.RTN_NORM_RMS, "layer": B.RTN_NORM_LAYER}
# one wave a row, four, eight; one, two and four pieces a lane; odd widths
SIZES = [(1, 1), (3, 7), (1, 64), (5, 511), (7, 513), (33, 1000), (2, 2049), (9, 4096), (4, 4100), (3, 8192), (2, 8200), (3, 16384), (600, 130)]


def rounded(dtype, v, e):
    return Q.U[dtype] * (np.abs(v) + e) + e + Q.STEP[dtype]


def norm64(v, kind, eps):
    """n(v), 1 / sqrt(..), and a bound of n's error in fp32"""
    C = v.shape[1]
    off = 0.0
    if kind == "layer":
        size = np.abs(v).mean(1, keepdims=True)
        v = v - v.mean(1, keepdims=True)
        off = (C + 2) * EPS * size
    r = 1 / np.sqrt((v * v).mean(1, keepdims=True) + eps)
    n = v * r
    # the variance takes on twice the mean's error times mean |v|, at most its root: n changes by n (off r)
    return n, r, (C / 2 + 8) * EPS * np.abs(n) + off * r * (1 + np.abs(n)) + EPS * np.abs(n)


def back64(dn, edn, n, en, r, kind):
    """r (dn - n mean(dn n) [- mean dn]) and a bound of its error, given those of dn and n (r's is within n's share of them)"""
    C = dn.shape[1]
    m = (dn * n).mean(1, keepdims=True)
    size = np.abs(dn * n).mean(1, keepdims=True)
    em = (C + 2) * EPS * size + (np.abs(dn) * en + edn * (np.abs(n) + en)).mean(1, keepdims=True)
    d, e = dn - n * m, edn + np.abs(n) * em + en * (np.abs(m) + em)
    total = np.abs(dn) + np.abs(n * m)
    if kind == "layer":
        mean = dn.mean(1, keepdims=True)
        d = d - mean
        ms = np.abs(dn).mean(1, keepdims=True)
        e = e + (C + 2) * EPS * ms + edn.mean(1, keepdims=True)
        total = total + ms
    # r itself: relative to r as n's error is to n, where n is of its own size 1
    er = en.max(1, keepdims=True)
    return d * r, r * (e * (1 + er) + er * total + 6 * EPS * total)


class Case:
    def __init__(self, dtype, M, C, kind, run=None, biases=True, gate=True, nxt=True, scale=0.75, seed=0, offset=0.3, eps=1e-5):
        rng = np.random.default_rng(seed + 100 * M + C)
        self.dtype, self.type, self.M, self.C, self.kind, self.scale, self.eps = dtype, Q.TYPES[dtype], M, C, kind, scale, eps
        self.run = run or M
        dev = lambda v: torch.from_numpy(np.ascontiguousarray(v, dtype=np.float32)).to(Q.DEV)
        self.h, self.x, self.dy, self.du = [(Q.values(rng, M, C, dtype).float() + offset * (i < 2)).to(self.type) for i in range(4)]
        self.weight, self.next_weight = dev(1 + 0.3 * rng.standard_normal(C)), dev(1 + 0.3 * rng.standard_normal(C)) if nxt else None
        self.bias, self.next_bias = (dev(0.2 * rng.standard_normal(C)), dev(0.2 * rng.standard_normal(C)) if nxt else None) if biases else (None, None)
        self.gate = dev(0.5 + 0.4 * rng.standard_normal((-(-M // self.run), C))) if gate else None

    def args(self):
        return dict(bias=self.bias, gate=self.gate, gate_run=self.run, scale=self.scale, kind=KINDS[self.kind], eps=self.eps)

    def vec(self, t, otherwise=0.0):
        return np.full(self.C, otherwise) if t is None else Q.f64(t)

    def owner(self):
        return np.arange(self.M) // self.run

    def gate64(self):
        return np.ones((self.M, self.C)) if self.gate is None else Q.f64(self.gate)[self.owner()]

    def post64(self):
        n, r, en = norm64(Q.f64(self.h), self.kind, self.eps)
        w, b = Q.f64(self.weight), self.vec(self.bias)
        p = n * w + b
        return n, r, en, p, en * np.abs(w) + 2 * EPS * (np.abs(n * w) + np.abs(b))


def check_forward(c, y, u):
    n, r, en, p, ep = c.post64()
    g, x = c.gate64(), Q.f64(c.x)
    want = c.scale * x + g * p
    T.assert_within(y, want, rounded(c.dtype, want, np.abs(g) * ep + 3 * EPS * (np.abs(g * p) + np.abs(c.scale * x))), "y")
    if u is not None:                                          # from y as it was rounded
        check_norm(c, y, c.next_weight, c.next_bias, u)


def check_norm(c, v, weight, bias, u):
    n, _, en = norm64(Q.f64(v), c.kind, c.eps)
    w, b = Q.f64(weight), c.vec(bias)
    want = n * w + b
    T.assert_within(u, want, rounded(c.dtype, want, en * np.abs(w) + 2 * EPS * (np.abs(n * w) + np.abs(b))), "u")


def check_sum(got, terms, eterms, axis_rows, what):
    want = terms.sum(0)
    T.assert_within(got, want, eterms.sum(0) + (axis_rows + 4) * EPS * (np.abs(terms) + eterms).sum(0) + EPS * np.abs(want), what)


def check_backward(c, got, y, dy=True, du=True):
    dh, dx, dweight, dbias, dgate, dnw, dnb = got
    d, ed = (Q.f64(c.dy), 0.0) if dy else (np.zeros((c.M, c.C)), 0.0)
    if du:
        n, r, en = norm64(Q.f64(y), c.kind, c.eps)
        g, w = Q.f64(c.du), Q.f64(c.next_weight)
        back, eb = back64(g * w, EPS * np.abs(g * w), n, en, r, c.kind)
        check_sum(dnw, g * n, np.abs(g) * en, c.M, "dnext_weight")
        check_sum(dnb, g, np.zeros_like(g), c.M, "dnext_bias")
        d, ed = d + back, eb + EPS * (np.abs(d) + np.abs(back))
    else:
        ed = np.zeros_like(d)
    want = c.scale * d
    T.assert_within(dx, want, rounded(c.dtype, want, abs(c.scale) * ed + EPS * np.abs(want)), "dx")
    n, r, en, p, ep = c.post64()
    g, w = c.gate64(), Q.f64(c.weight)
    dn = d * g * w
    back, eb = back64(dn, ed * np.abs(g * w) + 2 * EPS * np.abs(dn), n, en, r, c.kind)
    T.assert_within(dh, back, rounded(c.dtype, back, eb), "dh")
    # the sums over a run are formed of d n and d, multiplied by the gate or the weight afterwards
    terms, eterms = d * n, ed * (np.abs(n) + en) + np.abs(d) * en
    check_sum(dweight, g * terms, np.abs(g) * eterms, c.M, "dweight")
    if c.bias is not None or dbias is not None:
        check_sum(dbias, g * d, np.abs(g) * ed, c.M, "dbias")
    if c.gate is not None:
        b = c.vec(c.bias)
        for o in range(c.gate.shape[0]):
            m = c.owner() == o
            want = (d * p)[m].sum(0)
            bound = (np.abs(w) * eterms + np.abs(b) * ed)[m].sum(0) + (c.M + 6) * EPS * (np.abs(w) * (np.abs(terms) + eterms) + np.abs(b) * (np.abs(d) + ed))[m].sum(0)
            T.assert_within(dgate[o], want, bound, "dgate[%d]" % o)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("M,C", SIZES)
def test_norm(dtype, kind, M, C):
    c = Case(dtype, M, C, kind)
    u = B.norm(c.x, c.weight, bias=c.bias, kind=KINDS[kind], eps=c.eps)
    check_norm(c, c.x, c.weight, c.bias, u)
    dx, dw, db = B.norm_backward(c.du, c.x, c.weight, kind=KINDS[kind], eps=c.eps, dx_add=c.dy)
    n, r, en = norm64(Q.f64(c.x), kind, c.eps)
    g, w, a = Q.f64(c.du), Q.f64(c.weight), Q.f64(c.dy)
    back, eb = back64(g * w, EPS * np.abs(g * w), n, en, r, kind)
    T.assert_within(dx, a + back, rounded(dtype, a + back, eb + EPS * (np.abs(a) + np.abs(back))), "dx")
    check_sum(dw, g * n, np.abs(g) * en, M, "dweight")
    check_sum(db, g, np.zeros_like(g), M, "dbias")
    alone = B.norm_backward(c.du, c.x, c.weight, kind=KINDS[kind], eps=c.eps, want_dx=False, want_dbias=False)
    assert alone[0] is None and alone[2] is None and torch.equal(alone[1], dw)
    plain = B.norm_backward(c.du, c.x, c.weight, kind=KINDS[kind], eps=c.eps, want_dweight=False, want_dbias=False)[0]
    T.assert_within(plain, back, rounded(dtype, back, eb), "dx without the residual's")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("M,C", SIZES)
def test_block(dtype, kind, M, C):
    c = Case(dtype, M, C, kind, run=max(1, -(-M // 3)))
    y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
    check_forward(c, y, u)
    check_backward(c, B.block_norm_backward(c.dy, c.h, c.weight, du=c.du, y=y, next_weight=c.next_weight, **c.args()), y)


@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("biases,gate,nxt,dy", [(False, True, True, True), (True, False, True, True), (True, True, False, True), (False, False, False, True),
                                                (True, True, True, False)])
@pytest.mark.parametrize("M,C", [(1, 70), (50, 300), (20, 5000)])
def test_block_forms(kind, biases, gate, nxt, dy, M, C):
    c = Case("bf16", M, C, kind, biases=biases, gate=gate, nxt=nxt)
    y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
    assert (u is None) == (not nxt)
    check_forward(c, y, u)
    got = B.block_norm_backward(c.dy if dy else None, c.h, c.weight, du=c.du if nxt else None, y=y if nxt else None, next_weight=c.next_weight, **c.args())
    assert (got[4] is None) == (not gate) and (got[5] is None) == (not nxt) == (got[6] is None)
    check_backward(c, got, y, dy=dy, du=nxt)
    for i in range(7):                                         # each output alone
        if got[i] is None:
            continue
        want = {"want_" + k: i == j for j, k in enumerate(("dh", "dx", "dweight", "dbias", "dgate", "dnext_weight", "dnext_bias"))}
        one = B.block_norm_backward(c.dy if dy else None, c.h, c.weight, du=c.du if nxt else None, y=y if nxt else None, next_weight=c.next_weight, **c.args(), **want)
        assert torch.equal(one[i], got[i]) and all(one[j] is None for j in range(7) if j != i)


@pytest.mark.parametrize("run", [1, 2, 7, 299, 300, 1000])
def test_runs_of_the_gate(run):
    """A gate for every token, for runs that end inside and behind the tokens."""
    c = Case("bf16", 300, 200, "rms", run=run)
    y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
    check_forward(c, y, u)
    check_backward(c, B.block_norm_backward(c.dy, c.h, c.weight, du=c.du, y=y, next_weight=c.next_weight, **c.args()), y)


def test_many_rows():
    """More rows than units: each unit walks several, and a unit's sums are added up over them."""
    for M, C, run in ((9000, 40, 9000), (5000, 600, 1700)):
        c = Case("fp16", M, C, "layer", run=run)
        y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
        check_forward(c, y, u)
        check_backward(c, B.block_norm_backward(c.dy, c.h, c.weight, du=c.du, y=y, next_weight=c.next_weight, **c.args()), y)


@pytest.mark.parametrize("M,C", [(6, 205), (40, 3001)])
def test_rows_apart_and_in_place(M, C):
    c = Case("bf16", M, C, "layer")
    y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
    yo, uo = Q.apart(torch.zeros_like(y)), Q.apart(torch.zeros_like(y), 9, 5)
    B.block_norm(Q.apart(c.h), Q.apart(c.x), c.weight, next_weight=c.next_weight, next_bias=c.next_bias, y_out=yo, u_out=uo, **c.args())
    assert torch.equal(yo, y) and torch.equal(uo, u)
    assert (yo._base.view(-1)[1:].view(M, C + 3)[:, C:] == 7).all() and (uo._base.view(-1)[5:].view(M, C + 9)[:, C:] == 7).all()
    x, h = c.x.clone(), c.h.clone()
    B.block_norm(h, x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, y_out=x, u_out=h, **c.args())
    assert torch.equal(x, y) and torch.equal(h, u)
    got = B.block_norm_backward(c.dy, c.h, c.weight, du=c.du, y=y, next_weight=c.next_weight, **c.args())
    strided = B.block_norm_backward(Q.apart(c.dy), Q.apart(c.h), c.weight, du=Q.apart(c.du), y=Q.apart(y), next_weight=c.next_weight, **c.args())
    assert all(torch.equal(a, b) for a, b in zip(got, strided))
    un = B.norm(c.x, c.weight, kind=KINDS["layer"])
    xi = c.x.clone()
    B.norm(xi, c.weight, kind=KINDS["layer"], u_out=xi)
    assert torch.equal(xi, un)
    dx = B.norm_backward(c.du, c.x, c.weight, dx_add=c.dy)[0]
    acc = c.dy.clone()
    B.norm_backward(c.du, c.x, c.weight, dx_add=acc, dx=acc)
    assert torch.equal(acc, dx)


@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_gradients_against_differences(kind):
    """The 64-bit formulas that the library is held to above, against central differences of the forward formula."""
    rng = np.random.default_rng(3)
    M, C, run, scale, eps = 4, 6, 2, 0.7, 1e-5
    v = dict(h=rng.standard_normal((M, C)), x=rng.standard_normal((M, C)), w=rng.standard_normal(C), b=rng.standard_normal(C),
             g=rng.standard_normal((2, C)), nw=rng.standard_normal(C), nb=rng.standard_normal(C))
    dy, du = rng.standard_normal((M, C)), rng.standard_normal((M, C))

    def forward(v):
        y = scale * v["x"] + v["g"][np.arange(M) // run] * (norm64(v["h"], kind, eps)[0] * v["w"] + v["b"])
        return y, norm64(y, kind, eps)[0] * v["nw"] + v["nb"]

    loss = lambda v: (lambda y, u: (dy * y).sum() + (du * u).sum())(*forward(v))
    y, _ = forward(v)
    z = np.zeros((M, C))
    n2, r2, _ = norm64(y, kind, eps)
    d = dy + back64(du * v["nw"], z, n2, z, r2, kind)[0]
    n1, r1, _ = norm64(v["h"], kind, eps)
    g = v["g"][np.arange(M) // run]
    grads = dict(h=back64(d * g * v["w"], z, n1, z, r1, kind)[0], x=scale * d, w=(d * g * n1).sum(0), b=(d * g).sum(0),
                 g=(d * (n1 * v["w"] + v["b"])).reshape(2, run, C).sum(1), nw=(du * n2).sum(0), nb=du.sum(0))
    for k in v:
        for idx in np.ndindex(v[k].shape):
            step = 1e-5
            up, down = dict(v), dict(v)
            up[k], down[k] = v[k].copy(), v[k].copy()
            up[k][idx] += step
            down[k][idx] -= step
            diff = (loss(up) - loss(down)) / (2 * step)
            # the third derivative's share is of the order of step^2, the cancellation's 2^-53 / step
            assert abs(diff - grads[k][idx]) <= 1e-6 * (1 + abs(diff)), (k, idx)
    # and the library, in fp16, at the same point
    half = lambda a: torch.from_numpy(a.astype(np.float32)).to(Q.DEV).half()
    vec = lambda a: torch.from_numpy(a.astype(np.float32)).to(Q.DEV)
    kw = dict(gate=vec(v["g"]), gate_run=run, scale=scale, kind=KINDS[kind], eps=eps)
    yy, _ = B.block_norm(half(v["h"]), half(v["x"]), vec(v["w"]), bias=vec(v["b"]), next_weight=vec(v["nw"]), next_bias=vec(v["nb"]), **kw)
    got = B.block_norm_backward(half(dy), half(v["h"]), vec(v["w"]), bias=vec(v["b"]), du=half(du), y=yy, next_weight=vec(v["nw"]), **kw)
    for t, k in zip(got, ("h", "x", "w", "b", "g", "nw", "nb")):
        # inputs are off by 2^-11 of themselves, which rows of six values and 1 / sqrt(..) of up to a few units carry on some tens of times
        assert np.abs(Q.f64(t) - grads[k]).max() <= 64 * 2.0 ** -11 * max(1, np.abs(grads[k]).max()), k


def test_rows_of_zeros_and_values_that_are_not_finite():
    c = Case("bf16", 8, 100, "rms")
    for kind in ("rms", "layer"):
        x = c.x.clone()
        x[2] = 0
        x[3] = 5.0                                             # no variance
        x[5, 7] = float("inf")
        x[6, 99] = float("nan")
        u = B.norm(x, c.weight, bias=c.bias, kind=KINDS[kind])
        clean = B.norm(c.x, c.weight, bias=c.bias, kind=KINDS[kind])
        Q.equal(u[2], c.bias.to(u.dtype))
        if kind == "layer":
            Q.equal(u[3], c.bias.to(u.dtype))
        assert torch.isnan(u[6]).all() and torch.isnan(u[5, 7])
        for m in (0, 1, 4, 7):
            assert torch.equal(u[m], clean[m])
        assert torch.isfinite(B.norm_backward(c.du, x, c.weight, kind=KINDS[kind])[0][[0, 1, 2, 3, 4, 7]]).all()


def test_no_rows():
    c = Case("bf16", 4, 30, "rms")
    e = c.x[:0]
    assert B.norm(e, c.weight).shape == (0, 30)
    dx, dw, db = B.norm_backward(e, e, c.weight, dweight=torch.full((30,), 3.0, device=Q.DEV), dbias=torch.full((30,), 3.0, device=Q.DEV))
    assert dx.shape == (0, 30) and not dw.any() and not db.any()
    y, u = B.block_norm(e, e, c.weight, next_weight=c.weight)
    assert y.shape == u.shape == (0, 30)
    got = B.block_norm_backward(e, e, c.weight, du=e, y=y, next_weight=c.weight)
    assert got[0].shape == (0, 30) and not got[2].any() and not got[5].any()
    for gate in (torch.ones(30, device=Q.DEV), torch.ones((0, 30), device=Q.DEV)):
        y, _ = B.block_norm(e, e, c.weight, gate=gate, gate_run=4)
        dgate = B.block_norm_backward(e, e, c.weight, gate=gate, gate_run=4)[4]
        assert dgate.shape == gate.shape and not dgate.any()


def test_gate_runs_beyond_all_tokens():
    c = Case("bf16", 5, 60, "rms", gate=True)
    want = B.block_norm(c.h, c.x, c.weight, gate=c.gate, gate_run=5)[0]
    grad = B.block_norm_backward(c.dy, c.h, c.weight, gate=c.gate, gate_run=5)
    for run in (6, 1 << 40, (1 << 63) - 1):
        assert torch.equal(B.block_norm(c.h, c.x, c.weight, gate=c.gate, gate_run=run)[0], want)
        got = B.block_norm_backward(c.dy, c.h, c.weight, gate=c.gate.view(-1), gate_run=run)
        assert all(a is b is None or torch.equal(a.view(-1), b.view(-1)) for a, b in zip(got, grad))


def test_captured_and_on_two_streams():
    cs = [Case("bf16", 70, 900, "layer", run=30, seed=s) for s in (1, 2, 3)]

    def step(c):
        y, u = B.block_norm(c.h, c.x, c.weight, next_weight=c.next_weight, next_bias=c.next_bias, **c.args())
        return (y, u) + tuple(B.block_norm_backward(c.dy, c.h, c.weight, du=c.du, y=y, next_weight=c.next_weight, **c.args())) + \
            (B.norm(c.x, c.weight),) + tuple(B.norm_backward(c.du, c.x, c.weight))

    want = [step(c) for c in cs]
    torch.cuda.synchronize()
    hold = Case("bf16", 70, 900, "layer", run=30, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(hold)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(hold)
    for i in (1, 2, 0, 2):
        for k, t in vars(hold).items():
            if torch.is_tensor(t):
                t.copy_(getattr(cs[i], k))
        graph.replay()
        step(cs[0])
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want[i]))
    streams, got = [torch.cuda.Stream(), torch.cuda.Stream()], [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(step(cs[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(a, b) for g in got[i] for a, b in zip(g, want[i]))


def test_refusals_of_the_binding():
    c = Case("bf16", 6, 40, "rms")
    with pytest.raises(AssertionError):
        B.norm(c.x.float(), c.weight)
    with pytest.raises(AssertionError):
        B.norm(c.x, c.weight[:-1])
    with pytest.raises(AssertionError):
        B.norm(c.x, c.weight.bfloat16())
    with pytest.raises(AssertionError):
        B.block_norm(c.h, c.x[:-1], c.weight)
    with pytest.raises(AssertionError):
        B.block_norm(c.h, c.x, c.weight, gate=torch.ones((2, 40), device=Q.DEV))               # no gate_run
    with pytest.raises(AssertionError):
        B.block_norm(c.h, c.x, c.weight, gate=torch.ones((2, 40), device=Q.DEV), gate_run=2)   # three rows needed
    with pytest.raises(AssertionError):
        B.block_norm(c.h, c.x, c.weight, gate=torch.ones((4, 40), device=Q.DEV), gate_run=2)   # and no more
    with pytest.raises(AssertionError):
        B.block_norm(c.h, c.x, c.weight, gate=torch.ones((3, 40), device=Q.DEV), gate_run=0)
    with pytest.raises(B.RtnError) as e:
        B.norm(c.x, c.weight, eps=-1.0)
    assert e.value.status == B.RTN_ERR_SHAPE
    with pytest.raises(B.RtnError):
        B.norm(c.x, c.weight, kind=2)
    wide = torch.zeros((2, 16385), dtype=torch.bfloat16, device=Q.DEV)
    with pytest.raises(B.RtnError) as e:
        B.norm(wide, torch.ones(16385, device=Q.DEV))
    assert e.value.status == B.RTN_ERR_SHAPE
    with pytest.raises(B.RtnError) as e:
        B.block_norm_backward(None, c.h, c.weight)
    assert e.value.status == B.RTN_ERR_NULL
    need = B.lib().rtn_norm_backward_workspace_bytes(6, 40, 6)
    with pytest.raises(B.RtnError) as e:
        B.norm_backward(c.du, c.x, c.weight, workspace=torch.empty(need - 1, dtype=torch.uint8, device=Q.DEV))
    assert e.value.status == B.RTN_ERR_WORKSPACE
    with pytest.raises(ValueError):
        B.norm_backward(c.du, c.x, c.weight, workspace=torch.empty(need, dtype=torch.uint8))


@pytest.mark.parametrize("rows", [None, 0, 1, 3])
def test_rows_of_no_columns_are_refused(rows):
    """By every entry point, with and without a gate of no columns."""
    h, w = torch.empty((3, 0), dtype=torch.bfloat16, device=Q.DEV), torch.empty(0, device=Q.DEV)
    gate = {} if rows is None else dict(gate=torch.empty((rows, 0), device=Q.DEV) if rows else w, gate_run=1)
    for call in (lambda: B.norm(h, w), lambda: B.norm_backward(h, h, w), lambda: B.block_norm(h, h, w, next_weight=w, **gate),
                 lambda: B.block_norm_backward(h, h, w, **gate), lambda: B.block_norm_backward(h, h, w, want_dgate=False, **gate),
                 lambda: B.block_norm_backward(h, h, w, du=h, y=h, next_weight=w, **gate),
                 lambda: B.block_norm_backward(h[:0], h[:0], w, **gate)):
        with pytest.raises(B.RtnError) as e:
            call()
        assert e.value.status in (B.RTN_ERR_NULL, B.RTN_ERR_SHAPE)   # (an empty tensor has no address)
