"""Steps of every form that their rule takes: lanes along state_dim by its size, one or four wavefronts to a head, one to eight rounds of each."""
import pytest
import torch

import recur_ref
import test_gpu_recur as packed
from test_gpu_recur import srm  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("heads", [3, 40, 513])                # in all; few of them up to 512
@pytest.mark.parametrize("N,lanes", [(13, 4), (32, 8), (50, 16), (128, 32), (201, 64)])
@pytest.mark.parametrize("need", [1, 2, 3, 7, 8, 9, 16, 33, 70])    # rounds of a wavefront that P takes
def test_step(srm, need, N, lanes, heads, dtype):  # noqa: F811
    P, H, G = need * (64 // lanes) - (1 if need > 1 else 0), 3, 1
    rows = heads // H
    if rows * H * P * N > 1 << 25:
        pytest.skip("more than the reference should take")
    gen = torch.Generator().manual_seed(need * N)
    s = packed._heads(gen, rows, H, P, G, N, dtype, F32, z=need % 2 == 0)
    out, width = torch.empty(rows, H * P, dtype=dtype, device="cuda"), 2
    slot, pos = torch.randperm(rows, generator=gen).tolist(), torch.randint(0, 4, (rows,), generator=gen).tolist()
    if rows > 2:
        pos[1], slot[2] = -1, -1
    state, ring = torch.randn(rows, H, P, N, generator=gen).cuda(), torch.randn(rows, width, H * P + 2 * G * N, generator=gen).to(dtype).cuda()
    weight = torch.randn(H * P + 2 * G * N, width, generator=gen).cuda()
    held, held_ring = state.clone(), ring.clone()
    print(f"step {dtype}, {rows} rows of {H} heads {P} x {N}", flush=True)
    srm.selective_step(s["xbc"], s["dt"], s["a"], packed._i32(pos), state, out, groups=G, weight=weight, conv_state=ring, dt_bias=s["dt_bias"], skip=s["skip"],
                       z=s["z"], slot=packed._i32(slot))
    torch.cuda.synchronize()
    cpu = {k: v.cpu() if isinstance(v, torch.Tensor) else v for k, v in s.items()}
    off = list(range(rows + 1))
    conv, v, size, after_ring = recur_ref.conv(cpu["xbc"], weight.cpu(), None, off, pos, slot, held_ring.cpu())
    assert torch.equal(ring.double().cpu(), after_ring)
    wrong = recur_ref.conv_bound(conv, v, size, width, F32)
    kw = dict(offsets=off, H=H, P=P, G=G, N=N, pos=pos, slot=slot, state=held.cpu())
    want, mag, after, at = recur_ref.scan(**{**cpu, "xbc": conv}, **kw)
    _, up, _, up_state = recur_ref.scan(**{**cpu, "xbc": conv.abs() + wrong}, **kw)
    bound, of_state = recur_ref.scan_bounds(want, mag, at, 1, N, dtype, False)
    packed._near(out, want, bound + 1.01 * (up - mag), "out")
    packed._near(state, after, of_state + 1.01 * (up_state - at), "state")
