"""A feed-forward block of a language model with ternary weights, trained and served through the library:

    h = gelu(alpha1 * (x t1^T) + b1)        y = alpha2 * (h t2^T) + b2 + x

Latent fp32 weights w are ternarized every step (rtn_ternarize_pack, t = (w > 1/2) - (w < -1/2)) and laid out for both
directions (rtn_linear_prepare).  The forward pass keeps its input, the value before the activation and the second layer's
input in 8 bits (rtn_checkpoint_pack, rtn_linear's z_ckpt) and nothing in 16; the backward pass reads those
(rtn_linear_backward) and carries the gradient of alpha * t on to the latent weights and alpha (rtn_weight_backward: the
straight-through estimator clipped at |w| <= 1).  A model that answers lays the weights out once (`freeze`) and calls the
same layers for one token or many.

    python -m paper_1912_02057_amd.ternary_mlp      # trains against a teacher, then answers token by token
"""
import math

import torch

from . import binding as B

THRESHOLD = 0.5


class TernaryLinear:
    """One layer: latent weights [N, K], a scale and a bias per output."""

    def __init__(self, K, N, dtype=torch.bfloat16, device="cuda:0", generator=None):
        self.K, self.N, self.dtype = K, N, dtype
        self.w = 0.6 * torch.randn((N, K), generator=generator, device=device)
        self.alpha = torch.full((N,), 1.2 / math.sqrt(K), device=device)
        self.bias = torch.zeros(N, device=device)
        self._one, self._zero = torch.ones(N, device=device), torch.zeros(N, device=device)
        self.prepared = None

    def _codes(self):
        return B.ternarize_pack(self.w, -THRESHOLD, THRESHOLD, want_sum=False)[0]

    def freeze(self):
        """Lays the weights out for answering; latent weights changed afterwards need another call."""
        self.prepared = B.linear_prepare(self._codes(), self.N, self.K)
        self.bias16 = self.bias.to(self.dtype)

    def __call__(self, x, act=B.RTN_ACT_NONE, residual=None):
        return B.linear(x, self.prepared, self.N, self.alpha, bias=self.bias16, act=act, residual=residual)

    def forward(self, x, act=B.RTN_ACT_NONE, residual=None):
        """Of a training step: keeps x, and with an activation the value before it, in 8 bits."""
        self.act = act
        self.prepared, self.prepared_t = B.linear_prepare(self._codes(), self.N, self.K, backward=True)
        self.bias16 = self.bias.to(self.dtype)
        self.x8 = B.checkpoint_pack(x)
        self.z8 = None if act == B.RTN_ACT_NONE else B.checkpoint_empty(x.shape[0], self.N, x.device)
        return B.linear(x, self.prepared, self.N, self.alpha, bias=self.bias16, act=act, residual=residual, z_ckpt=self.z8)

    def backward(self, dy):
        """Gradients of the latent weights, alpha and the bias (kept) and of the input (returned)."""
        dx, dw, dbias = B.linear_backward(dy, self.prepared_t, self.K, self.alpha, self.x8, act=self.act, z_ckpt=self.z8,
                                          dw_dtype=torch.float32)
        self.x8 = self.z8 = self.prepared_t = None
        self.grad_w, sums = B.weight_backward(self.w, dw, -THRESHOLD, THRESHOLD, self._one, self._zero, self.alpha)
        self.grad_alpha, self.grad_bias = sums[:, 0].float(), dbias.float()
        return dx

    def step(self, rate):
        """Plain gradient descent; a weight's step is taken in its own unit, alpha."""
        self.w.sub_(self.grad_w / self.alpha[:, None] ** 2, alpha=rate)
        self.alpha.sub_(self.grad_alpha, alpha=0.01 * rate / self.K)
        self.bias.sub_(self.grad_bias, alpha=rate)


class TernaryMLP:
    def __init__(self, width, hidden, dtype=torch.bfloat16, device="cuda:0", seed=0):
        g = torch.Generator(device=device)
        g.manual_seed(seed)
        self.up = TernaryLinear(width, hidden, dtype, device, g)
        self.down = TernaryLinear(hidden, width, dtype, device, g)

    def freeze(self):
        self.up.freeze()
        self.down.freeze()
        return self

    def __call__(self, x):
        """[tokens, width] -> the same, weights as frozen."""
        return self.down(self.up(x, B.RTN_ACT_GELU), residual=x)

    def forward(self, x):
        return self.down.forward(self.up.forward(x, B.RTN_ACT_GELU), residual=x)

    def backward(self, dy):
        return self.up.backward(self.down.backward(dy)) + dy

    def step(self, rate):
        self.up.step(rate)
        self.down.step(rate)


def train(steps=60, tokens=512, width=256, hidden=1024, rate=0.02, seed=0, device="cuda:0"):
    """Fits a block to another one of fixed weights; returns the block and the losses (mean squares of the difference)."""
    teacher, block = TernaryMLP(width, hidden, device=device, seed=seed + 1).freeze(), TernaryMLP(width, hidden, device=device, seed=seed)
    g = torch.Generator(device=device)
    g.manual_seed(seed + 2)
    losses = []
    for _ in range(steps):
        x = torch.randn((tokens, width), generator=g, device=device).to(torch.bfloat16)
        diff = block.forward(x).float() - teacher(x).float()
        losses.append(diff.square().mean())
        block.backward((diff / tokens).to(torch.bfloat16))
        block.step(rate)
    return block, [float(v) for v in losses]


if __name__ == "__main__":
    block, losses = train()
    for i in range(0, len(losses), 10):
        print("step %3d  loss %.4f" % (i, losses[i]))
    print("last      loss %.4f" % losses[-1])
    block.freeze()
    x = torch.randn((64, 256), device="cuda:0").to(torch.bfloat16)
    at_once, one_by_one = block(x), torch.cat([block(x[i:i + 1]) for i in range(64)])
    print("64 tokens at once and one by one: largest difference %.3g of %.3g" % (float((at_once - one_by_one).abs().max()), float(at_once.abs().max())))
