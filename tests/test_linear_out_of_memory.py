"""Outputs that do not fit the device raise what torch raises, which callers catch to go on with less."""
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu


def test_out_of_memory_is_torchs_own_error():
    N = 1 << 21
    x = torch.zeros((1 << 20, 1), dtype=torch.bfloat16, device=T.DEV)
    w = torch.zeros(B.lib().rtn_linear_prepared_bytes(N, 1), dtype=torch.uint8, device=T.DEV)
    with pytest.raises(torch.OutOfMemoryError):
        B.linear(x, w, N, 1.0)                               # y: 4 TiB
    assert B.linear(x[:4], w, N, 1.0).shape == (4, N)        # and the next call is well
    torch.cuda.synchronize()
