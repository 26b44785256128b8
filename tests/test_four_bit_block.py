"""Norm, 4-bit layers, gate and residual run together, as a block of a language model uses them."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B
from paper_1912_02057_amd import ternary_mlp as M

import linear_testlib as T
import mx4_testlib as Q
from mx4_testlib import collected  # noqa: F401 (a fixture of the module)
from test_norm import back64, norm64, rounded

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("layer", [M.TernaryLinear, M.FourBitLinear])
@pytest.mark.parametrize("tokens,width,hidden", [(1, 96, 200), (70, 130, 257), (300, 256, 512)])
def test_the_block_is_its_parts(layer, tokens, width, hidden):
    """Forward and gradients of the block with norms: its ends against their formulas in 64 bits, on what the layers between them gave and
    were given; the layers have tests of their own."""
    block = M.TernaryMLP(width, hidden, seed=3, norm=True, layer=layer)
    rng = np.random.default_rng(4)
    for p in (block.w_in, block.w_out, block.gate):
        p.copy_(torch.from_numpy((1 + 0.3 * rng.standard_normal(width)).astype(np.float32)))
    x, dy = Q.values(rng, tokens, width, "bf16"), Q.values(rng, tokens, width, "bf16")
    seen = {}

    def spy(obj, name):
        call = getattr(obj, name)

        def wrapped(a, *args, **kw):
            out = call(a, *args, **kw)
            seen[obj, name] = (a.clone(), out.clone())
            return out
        setattr(obj, name, wrapped)
    for obj in (block.up, block.down):
        spy(obj, "forward")
        spy(obj, "backward")
    y = block.forward(x)
    dx = block.backward(dy)
    u, h = seen[block.up, "forward"][0], seen[block.down, "forward"][1]
    dh, du = seen[block.down, "backward"][0], seen[block.up, "backward"][1]
    x64, w_in, w_out, gate = Q.f64(x), Q.f64(block.w_in), Q.f64(block.w_out), Q.f64(block.gate)
    eps = 1e-6
    n, r, en = norm64(x64, "rms", eps)
    T.assert_within(u, n * w_in, rounded("bf16", n * w_in, (en + 2 * Q.EPS * np.abs(n)) * np.abs(w_in)), "u")
    m, s, em = norm64(Q.f64(h), "rms", eps)
    want = x64 + gate * (m * w_out)
    T.assert_within(y, want, rounded("bf16", want, np.abs(gate * w_out) * (em + 4 * Q.EPS * np.abs(m)) + 3 * Q.EPS * np.abs(x64)), "y")
    d = Q.f64(dy)
    back, eb = back64(d * gate * w_out, 2 * Q.EPS * np.abs(d * gate * w_out), m, em, s, "rms")
    T.assert_within(dh, back, rounded("bf16", back, eb), "dh")
    g = Q.f64(du)
    back, eb = back64(g * w_in, Q.EPS * np.abs(g * w_in), n, en, r, "rms")
    # the residual's gradient is dy, which is exact in its type
    T.assert_within(dx, d + back, rounded("bf16", d + back, eb + Q.EPS * (np.abs(d) + np.abs(back))), "dx")
    bound = lambda t, e: e.sum(0) + (tokens + 6) * Q.EPS * (np.abs(t) + e).sum(0)
    T.assert_within(block.grad_w_in, (g * n).sum(0), bound(g * n, np.abs(g) * en), "grad_w_in")
    T.assert_within(block.grad_w_out, (d * gate * m).sum(0), bound(d * gate * m, np.abs(d * gate) * em), "grad_w_out")
    T.assert_within(block.grad_gate, (d * m * w_out).sum(0), bound(d * m * w_out, np.abs(d * w_out) * em), "grad_gate")
    for obj, name in list(seen):
        delattr(obj, name)
    # answering runs the same calls
    block.freeze()
    one = torch.cat([block(x[i:i + 1]) for i in range(min(tokens, 5))])
    assert one.shape == (min(tokens, 5), width) and torch.isfinite(one.float()).all()


def test_four_bit_layers_gradients():
    """The layer of the block against the calls that it is made of, and its seed moves on."""
    L = M.FourBitLinear(70, 90, generator=torch.Generator(device=Q.DEV).manual_seed(1))
    x, dy = Q.values(np.random.default_rng(2), 40, 70, "bf16"), Q.values(np.random.default_rng(3), 40, 90, "bf16")
    before = int(L.seed)
    y = L.forward(x, B.RTN_ACT_GELU)
    dx = L.backward(dy)
    assert int(L.seed) == before + 1
    w, wt = B.mx4_pack(L.w, transposed=True)
    _, xt = B.mx4_pack(x, transposed=True)
    z = torch.empty_like(y)
    assert torch.equal(y, B.mx4_linear(x, w, 90, bias=L.bias16, act=B.RTN_ACT_GELU, z_out=z))
    want = B.mx4_linear_backward(dy, wt, 70, xt, act=B.RTN_ACT_GELU, z=z, seed=L.seed, dw_dtype=torch.float32)
    assert torch.equal(dx, want[0]) and torch.equal(L.grad_w, want[1]) and torch.equal(L.grad_bias, want[2].float())


@pytest.mark.parametrize("kw", [dict(norm=True), dict(layer=M.FourBitLinear), dict(norm=True, layer=M.FourBitLinear)])
def test_training_runs(kw):
    block, losses = M.train(steps=3, tokens=64, width=128, hidden=256, **kw)
    assert len(losses) == 3 and all(np.isfinite(losses))
