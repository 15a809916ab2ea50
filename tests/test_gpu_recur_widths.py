"""Every width of the short convolution, of prompts and in the step: filters whose window does not come round within a round of tokens, taps
beyond the third, positions on both sides of the width."""
import numpy as np
import pytest
import torch

import recur_ref
import test_gpu_recur as packed
from test_gpu_recur import srm  # noqa: F401

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [3, 5, 6, 7])
@pytest.mark.parametrize("channels,pad,offset", [(7, 2, 1), (13, 0, 3), (64, 8, 0), (333, 1, 1)])
def test_conv(srm, channels, pad, offset, width, dtype):  # noqa: F811
    packed.test_conv(srm, channels, pad, offset, width, dtype)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 2, 3, 4, 5, 6, 7, 8])
def test_conv_of_many_rows(srm, width, dtype):  # noqa: F811
    """As many wavefronts as take eight tokens at a time, whatever the width; sequences of several such rounds, and shorter ones."""
    gen = torch.Generator().manual_seed(width)
    channels, lengths = 4100, [1700, 3, 45, 0, 1, 2100]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    rows, n = int(off[-1]), len(lengths)
    x = torch.randn(rows, channels, generator=gen).to(dtype).cuda()
    weight, out = torch.randn(channels, width, generator=gen).cuda(), torch.empty_like(x)
    pos, slot = [0, 5, 2, 9, 0, 30], list(range(n))
    state = torch.randn(n, width, channels, generator=gen).to(dtype).cuda()
    held = state.clone()
    print(f"conv {dtype}, width {width}", flush=True)
    srm.causal_conv(x, weight, None, off, packed._i32(off.tolist()), out, pos=packed._i32(pos), slot=packed._i32(slot), state=state)
    torch.cuda.synchronize()
    want, v, size, after = recur_ref.conv(x.cpu(), weight.cpu(), None, off.tolist(), pos, slot, held.cpu())
    packed._near(out, want, recur_ref.conv_bound(want, v, size, width, dtype), "out")
    assert torch.equal(state.double().cpu(), after)


@pytest.mark.parametrize("dtype,dt_dtype,pad,offset", [(F32, F32, 0, 0), (BF16, F32, 3, 1)])
@pytest.mark.parametrize("H,P,G,N", [(2, 64, 1, 128), (8, 16, 4, 16), (3, 50, 1, 37), (2, 7, 2, 8), (1, 128, 1, 256)])
@pytest.mark.parametrize("width", [2, 3, 5, 6, 7, 8])
def test_step(srm, H, P, G, N, width, dtype, dt_dtype, pad, offset):  # noqa: F811
    packed.test_step(srm, H, P, G, N, width, dtype, dt_dtype, pad, offset)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [2, 3, 4, 5, 8])
def test_steps_from_the_first_token_are_the_convolution(srm, width, dtype):  # noqa: F811
    """Tokens 0 .. 2 width + 1 of a conversation one by one: what the ring holds, and what is taken of it, at every position."""
    gen = torch.Generator().manual_seed(width)
    H, P, G, N, T = 2, 20, 1, 12, 2 * width + 2
    C = H * P + 2 * G * N
    x = torch.randn(T, C, generator=gen).to(dtype)
    weight, bias = torch.randn(C, width, generator=gen), torch.randn(C, generator=gen)
    dt, a = 0.3 * torch.rand(T, H, generator=gen), -torch.rand(H, generator=gen)
    state, ring = torch.full((1, H, P, N), float("nan"), device="cuda"), torch.full((1, width, C), float("nan"), dtype=dtype, device="cuda")
    out, rows, sizes = torch.empty(T, H * P, dtype=dtype, device="cuda"), x.cuda(), dt.cuda()
    for t in range(T):
        srm.selective_step(rows[t:t + 1], sizes[t:t + 1], a.cuda(), packed._i32([t]), state, out[t:t + 1], weight=weight.cuda(), bias=bias.cuda(),
                           conv_state=ring, softplus=False)
    torch.cuda.synchronize()
    conv, v, size, _ = recur_ref.conv(x, weight, bias, [0, T], [0], [-1], None)
    wrong = recur_ref.conv_bound(conv, v, size, width, F32)
    kw = dict(dt=dt, a=a, offsets=[0, T], H=H, P=P, G=G, N=N, softplus=False, state=torch.zeros(1, H, P, N))
    want, mag, after, held = recur_ref.scan(conv, **kw)
    _, up, _, up_state = recur_ref.scan(conv.abs() + wrong, **kw)
    bound, of_state = recur_ref.scan_bounds(want, mag, held, T, N, dtype, False)
    packed._near(out, want, 1.05 * bound + 1.01 * (up - mag), "out")
    packed._near(state, after, 1.05 * of_state + 1.01 * (up_state - held), "state")
    last = torch.stack([x[p] for p in range(T)])
    for p in range(T - width, T):
        assert torch.equal(ring[0, p % width].cpu(), last[p])
