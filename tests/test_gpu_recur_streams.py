"""Scans on a stream of their own beside work that is queued on the current one."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_a_workspace_of_the_call_is_no_memory_that_queued_work_still_uses(srm, dtype):
    """The current stream's queued copy reads a block that the host has freed already, as long as the workspace of the scan that is launched
    meanwhile on another stream: both keep their results."""
    gen = torch.Generator().manual_seed(3)
    H, P, N, T = 2, 64, 128, 3000
    w = lambda cols: torch.randn(T, cols, generator=gen).to(dtype).cuda()  # noqa: E731
    xbc, dt, a = w(H * P + 2 * N), w(H), -torch.ones(H, device="cuda")
    off = np.array([0, T], dtype=np.int32)
    d_off = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    need = srm.selective_scan_workspace_bytes(srm.SRM_BF16 if dtype is BF16 else srm.SRM_FP32, off, H, P, N)
    assert need > 0
    want, got = (torch.empty(T, H * P, dtype=dtype, device="cuda") for _ in range(2))
    srm.selective_scan(xbc, dt, a, off, d_off, want)
    copied = torch.zeros(need, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    side = torch.cuda.Stream()
    block = torch.full((need,), 37, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    torch.cuda._sleep(20_000_000)                              # some 10 ms in front of the copy
    copied.copy_(block)
    del block
    for _ in range(3):
        srm.selective_scan(xbc, dt, a, off, d_off, got, stream=side)
    torch.cuda.synchronize()
    assert (copied == 37).all()
    assert torch.equal(got.view(torch.uint8), want.view(torch.uint8))
