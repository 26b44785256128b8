"""Values up to the end of the range that the layer takes: |x|, |dz| and their sums below 2^127 in bfloat16, all of float16's.  y and dx
are finite where alpha brings the sums back, and as exact as anywhere."""
import numpy as np
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu
END = {"bf16": 2.0 ** 127 * (1 - 2.0 ** -8), "fp16": 65504.0}


# a few tokens, small grids of aligned and of any rows, tiles; dx takes the same kernels over N
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("size", [(1, 64, 64), (7, 100, 1000), (3, 8200, 200), (40, 70, 1000), (40, 70, 333), (700, 1100, 328), (1100, 1000, 600), (2300, 2100, 264)])
def test_largest_values(dtype, size):
    M, N, K = size
    print("[case] largest values", dtype, size, flush=True)
    L = T.Layer(dtype, M, N, K, seed=M + N, residual=False)
    L.alpha = L.alpha * 2.0 ** -10
    rng = np.random.default_rng(K)

    def spread(t):
        """One element of a row at the end, or two whose sum and difference are below it, beside others of ordinary size."""
        v = T.f64(t)
        for m in range(v.shape[0]):
            at = rng.choice(v.shape[1], 2, replace=False) if v.shape[1] > 1 else [0]
            if m % 2:
                v[m, at] = END[dtype] / 2 * rng.choice([-0.99, 0.99], len(at))
            else:
                v[m, at[0]] = END[dtype] * rng.choice([-1, 1])
        return torch.from_numpy(v).to(L.type).to(T.DEV)
    L.x, L.dy = spread(L.x), spread(L.dy)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    y, e = L.y64("none")
    T.assert_within(B.linear(L.x, w, N, L.alpha, bias=L.bias), y, L.rounded(y, e), "y")
    for alpha in (2.0 ** -14, L.alpha):                      # dy as it is, and times alpha
        L.alpha = alpha
        dx = (T.f64(L.dy) * L.a64) @ L.t
        rounding = T.U[dtype] if torch.is_tensor(alpha) else 0.0
        ex = (rounding + (N + 3) * T.EPS) * (np.abs(T.f64(L.dy) * L.a64) @ np.abs(L.t))
        if dtype == "fp16":                                  # subnormal operands: test_linear_small_gradients.py
            ex = ex + N * 2.0 ** -38 * END[dtype] * np.abs(L.a64).max()
        got = B.linear_backward(L.dy, wt, K, alpha, None, want_dw=False, want_dbias=False)[0]
        T.assert_within(got, dx, L.rounded(dx, ex), "dx")
