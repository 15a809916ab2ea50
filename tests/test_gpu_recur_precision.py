"""What the selective scan, the step and the convolution may lose, against the same in 64 bits, token by token (recur_ref)."""
import numpy as np
import pytest
import torch

import recur_ref

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _over(got, want, bound):
    """By how much the worst element is outside its bound, and how many are."""
    got = got.double().cpu()
    assert torch.isfinite(got).all()
    over = (got - want).abs() - bound
    return float(over.max()), int((over > 0).sum())


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("H,P,G,N", [(4, 64, 1, 8), (2, 64, 1, 64), (2, 64, 2, 128), (2, 40, 1, 256), (3, 50, 1, 37)])
def test_a_scan_of_bf16_rounds_its_output_alone(srm, H, P, G, N, pad):
    """Beside the output's rounding nothing is kept in bf16: what is multiplied on the matrix cores is cut into two numbers at least: the upper
    half, which leaves less than a step (2^-7 of it), and what is left, rounded to half a step (2^-8 of that), so that 2^-15 of it is lost; a
    term of y is made of one such number (a weight of an earlier token, or an element of the state) and exact ones.  With one number
    instead of two the bound does not hold."""
    gen = torch.Generator().manual_seed(N + pad)
    off, n = [0, 33, 130], 130
    w = lambda cols: torch.randn(n, cols + pad, generator=gen).to(BF16).cuda()[:, :cols]  # noqa: E731
    xbc, z, dt = w(H * P + 2 * G * N), w(H * P), torch.rand(n, H, generator=gen).cuda()
    a, skip = -4.0 * torch.rand(H, generator=gen).cuda(), torch.zeros(H, device="cuda")
    state = torch.randn(2, H, P, N, generator=gen).cuda()
    held = state.cpu()
    out = torch.empty(n, H * P + pad, dtype=BF16, device="cuda")[:, :H * P]
    srm.selective_scan(xbc, dt, a, off, _i32(off), out, groups=G, skip=skip, z=z, softplus=False, pos=_i32([4, 0]), state=state)
    torch.cuda.synchronize()
    want, size, after, mag = recur_ref.scan(xbc.cpu(), dt.cpu(), a.cpu(), off, H, P, G, N, skip=skip.cpu(), z=z.cpu(), softplus=False, pos=[4, 0], state=held)
    bound, of_state = recur_ref.scan_bounds(want, size, mag, 97, N, BF16, False)
    worst, many = _over(out, want, bound + 2.0 ** -15 * 1.02 * size)
    print(f"{H} x {P}, {N}: error {float((out.double().cpu() - want).norm() / want.norm()):.3e} of the norm, rounding alone "
          f"{float((want.to(BF16).double() - want).norm() / want.norm()):.3e}; {many} outside", flush=True)
    assert many == 0, worst
    assert _over(state, after, of_state)[1] == 0
