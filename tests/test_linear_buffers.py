"""What the binding says to buffers that the kernels cannot take, and when the device's memory does not suffice."""
import pytest
import torch

from paper_1912_02057_amd import binding as B

import linear_testlib as T

pytestmark = pytest.mark.gpu


def test_workspaces_are_device_buffers():
    """A given workspace is used only if the kernels may write all of it: on the device, dense and large enough."""
    M, N, K = 2100, 1030, 131                                # odd rows into tiles: a workspace of M x 192 elements
    L = T.Layer("bf16", M, N, K, seed=1)
    w, wt = B.linear_prepare(L.codes, N, K, backward=True)
    x8 = B.checkpoint_pack(L.x)
    need = B.lib().rtn_linear_workspace_bytes(L.x.data_ptr(), K, M, N, K, 0)
    back = B.lib().rtn_linear_backward_workspace_bytes(M, N, K)
    assert need == M * 192 * 2 and back > 0
    forward = lambda ws: B.linear(L.x, w, N, L.alpha, workspace=ws)
    backward = lambda ws: B.linear_backward(L.dy, wt, K, L.alpha, x8, workspace=ws)
    for call, size in ((forward, need), (backward, back)):
        for bad in (torch.empty(size, dtype=torch.uint8),                              # the host's
                    torch.empty(2 * size, dtype=torch.uint8, device=T.DEV)[::2],       # with gaps
                    torch.empty(1, dtype=torch.uint8, device=T.DEV).expand(size)):     # one byte
            with pytest.raises(ValueError):
                call(bad)
        with pytest.raises(B.RtnError) as e:
            call(torch.empty(size - 1, dtype=torch.uint8, device=T.DEV))
        assert e.value.status == B.RTN_ERR_WORKSPACE
    good = torch.empty(need + 256, dtype=torch.uint8, device=T.DEV)
    assert torch.equal(forward(good), forward(None))
    good = torch.empty(back + 256, dtype=torch.uint8, device=T.DEV)
    assert all(torch.equal(a, b) for a, b in zip(backward(good), backward(None)))
