"""The short convolution, the selective scan of packed prompts and the step of single tokens through the public binding, against the same
in 64 bits, token by token (recur_ref, which derives the bounds)."""
import math

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


def _wide(gen, rows, cols, pad, dtype, offset=0, scale=1.0):
    """rows x cols inside a wider array that begins at any element."""
    flat = (torch.randn(offset + rows * (cols + pad), generator=gen) * scale).to(dtype).cuda()
    return flat[offset:].view(rows, cols + pad)[:, :cols]


def _i32(v):
    return None if v is None else torch.tensor(v, dtype=torch.int32, device="cuda")


def _near(got, want, bound, what):
    got = got.double().cpu()
    assert torch.isfinite(got).all(), what
    over = (got - want).abs() - bound
    assert (over <= 0).all(), (what, float(over.max()), int(over.argmax()), float((got - want).abs().max()))


# ------------------------------------------------------------------ convolution
LENGTHS = [[1], [0, 1, 2, 0, 3, 4, 5], [8], [7, 9], [100], [1, 1, 1, 1, 1, 30, 1, 64], [65, 0, 17], [3] * 90, [1] * 70, [2, 1, 0] * 30]


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("width", [1, 2, 4, 8])
@pytest.mark.parametrize("channels,pad,offset", [(1, 0, 0), (7, 2, 1), (8, 0, 0), (13, 0, 3), (64, 8, 0), (333, 1, 1), (512, 0, 0), (1100, 4, 0)])
def test_conv(srm, channels, pad, offset, width, dtype):
    gen = torch.Generator().manual_seed(channels * 10 + width)
    for lengths in LENGTHS:
        first, behind = 3, 5                                   # rows that belong to no sequence
        off = (first + np.concatenate([[0], np.cumsum(lengths)])).astype(np.int32)
        rows, n = int(off[-1]) + behind, len(lengths)
        x = _wide(gen, rows, channels, pad, dtype, offset)
        out = _wide(gen, rows, channels, pad, dtype, offset)
        before = out.clone()
        weight, bias = torch.randn(channels, width, generator=gen).cuda(), torch.randn(channels, generator=gen).cuda()
        slots = n + 2
        slot = torch.randperm(slots, generator=gen)[:n].tolist()
        pos = torch.randint(0, 12, (n,), generator=gen).tolist()
        if n > 2:
            slot[1], slot[2], pos[n // 2] = -1, slots, -3       # nothing kept, nothing kept, idle
        state = torch.randn(slots, width, channels, generator=gen).to(dtype).cuda()
        held = state.clone()
        activation = len(lengths) % 2 == 1
        print(f"conv {dtype} {channels} channels, width {width}, lengths {lengths}", flush=True)
        srm.causal_conv(x, weight, bias if activation else None, off, _i32(off.tolist()), out, pos=_i32(pos), slot=_i32(slot), state=state,
                        activation=activation)
        torch.cuda.synchronize()
        want, v, size, after = recur_ref.conv(x.cpu(), weight.cpu(), bias.cpu() if activation else None, off.tolist(), pos, slot, held.cpu(), activation)
        lo, hi = int(off[0]), int(off[-1])
        assert torch.equal(out[:lo], before[:lo]) and torch.equal(out[hi:], before[hi:])
        _near(out[lo:hi], want[lo:hi], recur_ref.conv_bound(want, v, size, width, dtype, activation)[lo:hi], (lengths, "out"))
        assert torch.equal(state.double().cpu(), after)


def test_conv_in_parts_is_conv_of_the_whole(srm):
    """A prompt in several calls, through the ring, gives the bits of one call; without a state all sequences start from zeros."""
    gen = torch.Generator().manual_seed(5)
    T, C, W = 150, 200, 4
    x, weight = _wide(gen, T, C, 0, BF16), torch.randn(C, W, generator=gen).cuda()
    whole = torch.empty_like(x)
    off = [0, T]
    srm.causal_conv(x, weight, None, off, _i32(off), whole)
    state = torch.full((3, W, C), math.nan, dtype=BF16, device="cuda")          # position 0 reads nothing of it
    parts = torch.empty_like(x)
    at = 0
    for n in (1, 1, 2, 50, 1, 95):
        off = [at, at + n]
        srm.causal_conv(x, weight, None, off, _i32(off), parts, pos=_i32([at]), slot=_i32([2]), state=state)
        at += n
    torch.cuda.synchronize()
    assert at == T and torch.equal(whole, parts)


# ------------------------------------------------------------------ scan
HEADS = [(2, 64, 1, 128), (4, 64, 2, 64), (3, 50, 1, 37), (8, 16, 4, 16), (1, 128, 1, 256), (2, 1, 1, 1), (2, 7, 2, 8), (6, 40, 3, 200), (2, 64, 2, 32),
         (1, 200, 1, 96)]
RUNS = [[1], [0, 1, 2, 0, 63], [64, 65], [17, 128, 1, 5], [300], [15, 16, 17, 33], [700, 0, 90, 3]]


def _heads(gen, rows, H, P, G, N, dtype, dt_dtype, pad=0, offset=0, z=True):
    s = dict(dt_bias=torch.randn(H, generator=gen).cuda() - 2, skip=torch.randn(H, generator=gen).cuda())
    s["a"] = -torch.exp(torch.randn(H, generator=gen)).cuda()
    s["xbc"] = _wide(gen, rows, H * P + 2 * G * N, pad, dtype, offset)
    s["dt"] = _wide(gen, rows, H, pad, dt_dtype, offset)
    s["z"] = _wide(gen, rows, H * P, pad, dtype, offset) if z else None
    return s


def _cpu(s, *but):
    return {k: v.cpu() if isinstance(v, torch.Tensor) else v for k, v in s.items() if k not in but}


@pytest.mark.parametrize("dtype,dt_dtype,pad,offset", [(F32, F32, 0, 0), (F32, BF16, 5, 1), (BF16, BF16, 0, 0), (BF16, F32, 3, 1), (BF16, BF16, 8, 8)])
@pytest.mark.parametrize("H,P,G,N", HEADS)
def test_scan(srm, H, P, G, N, dtype, dt_dtype, pad, offset):
    gen = torch.Generator().manual_seed(H * P + N + pad)
    for k, lengths in enumerate(RUNS):
        first, behind = 2, 3
        off = (first + np.concatenate([[0], np.cumsum(lengths)])).astype(np.int32)
        rows, n = int(off[-1]) + behind, len(lengths)
        s = _heads(gen, rows, H, P, G, N, dtype, dt_dtype, pad, offset, z=k % 3 != 1)
        if k % 3 == 2:
            s["skip"] = None
        out = _wide(gen, rows, H * P, pad, dtype, offset)
        before = out.clone()
        slots = n + 2
        slot = torch.randperm(slots, generator=gen)[:n].tolist()
        pos = torch.randint(0, 3, (n,), generator=gen).tolist()
        pos[-1] = 7
        if n > 3:
            slot[2], pos[0], pos[3] = -1, -1, 0
        state = torch.randn(slots, H, P, N, generator=gen).cuda()
        held = state.clone()
        print(f"scan {dtype} dt {dt_dtype} heads {H} x {P}, groups {G}, state {N}, lengths {lengths}, pad {pad}", flush=True)
        srm.selective_scan(s["xbc"], s["dt"], s["a"], off, _i32(off.tolist()), out, groups=G, dt_bias=s["dt_bias"], skip=s["skip"], z=s["z"],
                           pos=_i32(pos), slot=_i32(slot), state=state)
        torch.cuda.synchronize()
        want, size, after, mag = recur_ref.scan(offsets=off.tolist(), H=H, P=P, G=G, N=N, pos=pos, slot=slot, state=held.cpu(), **_cpu(s))
        lo, hi = int(off[0]), int(off[-1])
        assert torch.equal(out[:lo], before[:lo]) and torch.equal(out[hi:], before[hi:])
        bound, of_state = recur_ref.scan_bounds(want, size, mag, max(lengths), N, dtype, dtype is BF16)
        _near(out[lo:hi], want[lo:hi], bound[lo:hi], (lengths, "out"))
        _near(state, after, of_state, (lengths, "state"))
        for i in set(range(slots)) - {slot[j] for j in range(n) if pos[j] >= 0 and lengths[j]}:
            assert torch.equal(state[i], held[i])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_scan_without_state_softplus_or_bias(srm, dtype):
    gen = torch.Generator().manual_seed(3)
    H, P, G, N, off = 4, 64, 1, 64, [0, 70, 71, 330]
    s = _heads(gen, off[-1], H, P, G, N, dtype, F32, z=False)
    s["dt"] = s["dt"].abs() * 0.2
    s["dt_bias"] = s["skip"] = None
    out = torch.empty(off[-1], H * P, dtype=dtype, device="cuda")
    srm.selective_scan(s["xbc"], s["dt"], s["a"], off, _i32(off), out, softplus=False)
    torch.cuda.synchronize()
    want, size, _, _ = recur_ref.scan(offsets=off, H=H, P=P, G=G, N=N, softplus=False, **_cpu(s))
    bound, _ = recur_ref.scan_bounds(want, size, size, 260, N, dtype, dtype is BF16)
    _near(out, want, bound, "out")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("room", [0, 1, 2, 3, 5])
def test_scan_with_less_workspace_than_it_asks_for(srm, dtype, room):
    """Room for any number of segments, none among them."""
    gen = torch.Generator().manual_seed(room)
    H, P, G, N = 2, 64, 1, 128
    off = np.array([0, 900, 901, 1500], dtype=np.int32)
    s = _heads(gen, 1500, H, P, G, N, dtype, dtype)
    state = torch.randn(3, H, P, N, generator=gen).cuda()
    held = state.clone()
    out = torch.empty(1500, H * P, dtype=dtype, device="cuda")
    one = (2 * P * N + 1) * H * 4
    full = srm.selective_scan_workspace_bytes(1 if dtype is BF16 else 0, off, H, P, N)
    assert full % one == 0 and full >= 5 * one
    ws = torch.empty(room * one + 3, dtype=torch.uint8, device="cuda")
    srm.selective_scan(s["xbc"], s["dt"], s["a"], off, _i32(off.tolist()), out, dt_bias=s["dt_bias"], skip=s["skip"], z=s["z"], pos=_i32([5, 5, 0]),
                       state=state, workspace=ws)
    torch.cuda.synchronize()
    want, size, after, mag = recur_ref.scan(offsets=off.tolist(), H=H, P=P, G=G, N=N, pos=[5, 5, 0], state=held.cpu(), **_cpu(s))
    bound, of_state = recur_ref.scan_bounds(want, size, mag, 900, N, dtype, dtype is BF16)
    _near(out, want, bound, "out")
    _near(state, after, of_state, "state")


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T", [50, 400])
def test_what_is_not_finite_stays_behind_its_token_in_its_channel(srm, dtype, T):
    """An infinite or NaN x at a token leaves the outputs in front of it, other channels, other heads and other sequences as they are."""
    gen = torch.Generator().manual_seed(T)
    H, P, G, N = 2, 64, 1, 64
    off = [0, T, T + 40]
    s = _heads(gen, T + 40, H, P, G, N, dtype, F32)
    clean, dirty = (torch.empty(T + 40, H * P, dtype=dtype, device="cuda") for _ in range(2))
    st = [torch.zeros(2, H, P, N, device="cuda") for _ in range(2)]
    kw = dict(dt_bias=s["dt_bias"], skip=s["skip"], z=s["z"])
    srm.selective_scan(s["xbc"], s["dt"], s["a"], off, _i32(off), clean, state=st[0], **kw)
    bad = s["xbc"].clone()
    for at, p, value in ((37, 5, math.nan), (20, 70, math.inf), (41, 99, -math.inf)):
        bad[at, p] = value
    srm.selective_scan(bad, s["dt"], s["a"], off, _i32(off), dirty, state=st[1], **kw)
    torch.cuda.synchronize()
    touched = torch.zeros(T + 40, H * P, dtype=torch.bool, device="cuda")
    touched[37:T, 5] = touched[20:T, 70] = touched[41:T, 99] = True
    assert torch.equal(dirty[~touched], clean[~touched])
    assert not torch.isfinite(dirty[touched]).any()
    rows = torch.zeros(2, H, P, dtype=torch.bool, device="cuda")
    rows[0, 0, 5] = rows[0, 1, 6] = rows[0, 1, 35] = True
    assert torch.equal(st[1][~rows], st[0][~rows]) and not torch.isfinite(st[1][rows]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_decays_that_leave_nothing_and_step_sizes_of_any_size(srm, dtype):
    """Steps so long that a decay is 0 in fp32 among ordinary ones: what comes behind them does not lose digits."""
    gen = torch.Generator().manual_seed(8)
    H, P, G, N, T = 2, 32, 1, 32, 330
    s = _heads(gen, T, H, P, G, N, dtype, F32, z=False)
    s["dt"] = 0.05 * torch.rand(T, H, generator=gen).cuda()
    s["dt"][3::29] = 300.0
    s["dt"][10::37, 1] = 1e30
    s["dt"][5::41] = 0.0
    s["a"] = torch.tensor([-0.5, -20.0], device="cuda")
    s["xbc"][3::29] = s["xbc"][3::29] * 1e-3
    s["xbc"][10::37, P:2 * P] = 0.0
    s["dt_bias"] = None
    off = [0, T]
    out, state = torch.empty(T, H * P, dtype=dtype, device="cuda"), torch.randn(1, H, P, N, generator=gen).cuda()
    held = state.cpu()
    srm.selective_scan(s["xbc"], s["dt"], s["a"], off, _i32(off), out, skip=s["skip"], softplus=False, pos=_i32([1]), state=state)
    torch.cuda.synchronize()
    want, size, after, mag = recur_ref.scan(offsets=off, H=H, P=P, G=G, N=N, softplus=False, pos=[1], state=held, **_cpu(s))
    bound, of_state = recur_ref.scan_bounds(want, size, mag, T, N, dtype, dtype is BF16)
    _near(out, want, bound, "out")
    _near(state, after, of_state, "state")


# ------------------------------------------------------------------ single tokens
@pytest.mark.parametrize("dtype,dt_dtype,pad,offset", [(F32, F32, 0, 0), (BF16, BF16, 0, 0), (BF16, F32, 3, 1)])
@pytest.mark.parametrize("H,P,G,N", HEADS)
@pytest.mark.parametrize("width", [0, 1, 4])
def test_step(srm, H, P, G, N, width, dtype, dt_dtype, pad, offset):
    gen = torch.Generator().manual_seed(H * P + N + width)
    C = H * P + 2 * G * N
    for B in (1, 6):
        s = _heads(gen, B, H, P, G, N, dtype, dt_dtype, pad, offset, z=B > 1)
        out = _wide(gen, B, H * P, pad, dtype, offset)
        slots = B + 2
        slot, pos = torch.randperm(slots, generator=gen)[:B].tolist(), torch.randint(1, 9, (B,), generator=gen).tolist()
        if B > 1:
            pos[0], pos[1], slot[2], slot[3] = 0, -1, -1, slots
        state = torch.randn(slots, H, P, N, generator=gen).cuda()
        weight = torch.randn(C, width, generator=gen).cuda() if width else None
        bias = torch.randn(C, generator=gen).cuda() if width else None
        ring = torch.randn(slots, max(1, width), C, generator=gen).to(dtype).cuda()
        held, held_ring = state.clone(), ring.clone()
        print(f"step {dtype} dt {dt_dtype} heads {H} x {P}, groups {G}, state {N}, width {width}, {B} rows", flush=True)
        srm.selective_step(s["xbc"], s["dt"], s["a"], _i32(pos), state, out, groups=G, weight=weight, bias=bias, conv_state=ring if width else None,
                           dt_bias=s["dt_bias"], skip=s["skip"], z=s["z"], slot=_i32(slot))
        torch.cuda.synchronize()
        cpu, off = _cpu(s), list(range(B + 1))
        rows, wrong = cpu["xbc"].double(), 0.0
        if width:
            rows, v, size, after_ring = recur_ref.conv(cpu["xbc"], weight.cpu(), bias.cpu(), off, pos, slot, held_ring.cpu())
            assert torch.equal(ring.double().cpu(), after_ring)
            wrong = recur_ref.conv_bound(rows, v, size, width, F32)
        else:
            assert torch.equal(ring, held_ring)
        cpu["xbc"] = rows
        want, size, after, mag = recur_ref.scan(offsets=off, H=H, P=P, G=G, N=N, pos=pos, slot=slot, state=held.cpu(), **cpu)
        bound, of_state = recur_ref.scan_bounds(want, size, mag, 1, N, dtype, False)
        if width:                                              # what the convolution's error makes of the sums: all of x, B and C moved up by it
            cpu["xbc"] = rows.abs() + wrong
            _, up, _, up_state = recur_ref.scan(offsets=off, H=H, P=P, G=G, N=N, pos=pos, slot=slot, state=held.cpu(), **cpu)
            bound, of_state = bound + 1.01 * (up - size), of_state + 1.01 * (up_state - mag)
        _near(out, want, bound, "out")
        _near(state, after, of_state, "state")
        for i in set(range(slots)) - {slot[j] for j in range(B) if pos[j] >= 0}:
            assert torch.equal(state[i], held[i])


# ------------------------------------------------------------------ far addresses
def test_rows_slots_and_strides_beyond_32_bits(srm):
    gen = torch.Generator().manual_seed(1)
    H, P, G, N, W = 2, 32, 1, 32, 4
    C = H * P + 2 * G * N
    ld = (1 << 30) + 8
    far = torch.empty(3 * ld, dtype=BF16, device="cuda").as_strided((3, C), (ld, 1))
    rows = torch.randn(3, C, generator=gen).to(BF16).cuda()
    far.copy_(rows)
    weight = torch.randn(C, W, generator=gen).cuda()
    near, far_out = torch.empty_like(rows), torch.empty(3 * ld, dtype=BF16, device="cuda").as_strided((3, C), (ld, 1))
    off = [0, 3]
    srm.causal_conv(rows, weight, None, off, _i32(off), near)
    srm.causal_conv(far, weight, None, off, _i32(off), far_out)
    torch.cuda.synchronize()
    assert torch.equal(near, far_out)
    del far_out
    dt, a = torch.randn(3, H, generator=gen).cuda(), -torch.ones(H, device="cuda")
    out, out2 = torch.empty(3, H * P, dtype=BF16, device="cuda"), torch.empty(3, H * P, dtype=BF16, device="cuda")
    slots = (1 << 31) // (H * P * N) + 2
    state = torch.empty(slots, H, P, N, device="cuda")
    small = torch.zeros(1, H, P, N, device="cuda")
    srm.selective_scan(rows, dt, a, off, _i32(off), out, state=small)
    srm.selective_scan(far, dt, a, off, _i32(off), out2, slot=_i32([slots - 1]), state=state)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(state[-1], small[0])
    ring, ring1 = torch.zeros(slots, W, C, dtype=BF16, device="cuda"), torch.zeros(1, W, C, dtype=BF16, device="cuda")
    step = dict(weight=weight, activation=True)
    srm.selective_step(rows[2:], dt[2:], a, _i32([3]), small, out[2:], conv_state=ring1, **step)
    srm.selective_step(far[2:], dt[2:], a, _i32([3]), state, out2[2:], conv_state=ring, slot=_i32([slots - 1]), **step)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(state[-1], small[0]) and torch.equal(ring[-1], ring1[0])
