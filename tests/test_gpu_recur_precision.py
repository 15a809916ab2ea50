"""What the selective scan, the step and the convolution may lose, against the same in 64 bits, token by token (recur_ref)."""
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


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("entry", ["scan", "step"])
def test_step_sizes_to_an_ulp_or_two(srm, entry, dtype):
    """x = B = 1 from an empty state leave dt itself in the state.  The exponential loses an ulp at most (2^-23), the logarithm two, their sum with
    v half of one; cut into three numbers of bf16 and added up in fp32, an ulp more.  (Of these three, one below 2^-126 is a subnormal number, which the matrix
    cores take as 0: what is left of dt when the first one, or the first two, are taken off it is less than 2^-126 then, and so is the loss.
    It shows at dt = 1e-37.)"""
    H = 4096
    v = torch.cat([torch.linspace(-85, 40, 3 * H), torch.linspace(-12, 0, 6 * H), torch.linspace(-3.2, -2.4, 2 * H), torch.linspace(-0.8, 0.8, H)]).float()
    a, off = -torch.ones(H, device="cuda"), [0, 1]
    ones = torch.ones(1, H + 2, dtype=dtype, device="cuda")
    got = []
    for part in v.view(-1, 1, H):
        state, out = torch.full((1, H, 1, 1), 7.0, device="cuda"), torch.empty(1, H, dtype=dtype, device="cuda")
        if entry == "scan":
            srm.selective_scan(ones, part.cuda(), a, off, _i32(off), out, state=state)
        else:
            srm.selective_step(ones, part.cuda(), a, _i32([0]), state, out)
        got.append(state.view(-1))
    torch.cuda.synchronize()
    got, want = torch.cat(got).double().cpu(), recur_ref.sizes(v, None, True)
    wrong = ((got - want).abs() - (2.0 ** -126 if dtype is BF16 and entry == "scan" else 0.0)).clamp_min(0) / want
    print(f"{entry} {dtype}: {float(wrong.max()):.2e} at {float(v[wrong.argmax()]):.4f}", flush=True)
    assert wrong.max() <= 2.0 ** -23 + 2.0 ** -22 + 2.0 ** -24 + 2.0 ** -23


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("entry", ["scan", "step"])
def test_decays_to_an_ulp_or_two(srm, entry, dtype):
    """x = 0 leaves the decay itself in a state of ones.  The exponent is a product in 64 bits in two parts of fp32 (2^-48 of it is lost), the
    exponential loses an ulp (2^-23), the second part's product and sum one between them, the state's product half of one."""
    H = 4096
    e = torch.cat([torch.linspace(-85, 0, 3 * H), torch.linspace(-2, 0, H)]).float()
    gen = torch.Generator().manual_seed(1)
    dt = torch.exp(torch.randn(e.numel(), generator=gen))
    a = e / dt
    got = []
    for k in range(0, e.numel(), H):
        part, factor = dt[None, k:k + H].cuda(), a[k:k + H].cuda()
        zeros = torch.zeros(1, H + 2, dtype=dtype, device="cuda")
        state, out = torch.ones(1, H, 1, 1, device="cuda"), torch.empty(1, H, dtype=dtype, device="cuda")
        if entry == "scan":
            srm.selective_scan(zeros, part, factor, [0, 1], _i32([0, 1]), out, softplus=False, pos=_i32([1]), state=state)
        else:
            srm.selective_step(zeros, part, factor, _i32([1]), state, out, softplus=False)
        got.append(state.view(-1))
    torch.cuda.synchronize()
    got, want = torch.cat(got).double().cpu(), torch.exp(dt.double() * a.double())
    wrong = (got - want).abs() / want
    print(f"{entry} {dtype}: {float(wrong.max()):.2e} at {float(e[wrong.argmax()]):.4f}", flush=True)
    assert wrong.max() <= 2.5 * 2.0 ** -23


@pytest.mark.parametrize("many", [1, 12, 24, 30])
def test_large_exponents_take_no_digits_of_the_weights_behind_them(srm, many):
    """`many` tokens of a block whose decays are 0, then ordinary ones whose terms nearly cancel in y, so that an error of the weights shows
    beside the output's rounding."""
    gen = torch.Generator().manual_seed(many)
    H, P, N, T = 4, 64, 8, 64
    xbc = torch.zeros(T, H * P + 2 * N)
    xbc[:, H * P:] = 1.0
    sign = torch.where(torch.rand(H * P, generator=gen) < 0.5, -1.0, 1.0)
    for t in range(many, T):
        xbc[t, :H * P] = sign if (t - many) % 2 else -sign
    dt = torch.ones(T, H)
    dt[:many] = 1e6
    a = -0.002 - 0.003 * torch.rand(H, generator=gen)
    xbc, out = xbc.to(BF16), torch.empty(T, H * P, dtype=BF16, device="cuda")
    state = torch.zeros(1, H, P, N, device="cuda")
    srm.selective_scan(xbc.cuda(), dt.cuda(), a.cuda(), [0, T], _i32([0, T]), out, softplus=False, state=state)
    torch.cuda.synchronize()
    want, size, after, mag = recur_ref.scan(xbc, dt, a, [0, T], H, P, 1, N, softplus=False, state=torch.zeros(1, H, P, N))
    bound, of_state = recur_ref.scan_bounds(want, size, mag, T - many, N, BF16, False)
    assert _over(out, want, bound + 2.0 ** -15 * 1.02 * size)[1] == 0
    assert _over(state, after, of_state)[1] == 0


@pytest.mark.parametrize("entry", ["conv", "gate of the scan", "gate of the step", "step fp32", "step bf16"])
def test_silu_of_what_stays_in_fp32_to_a_few_ulp(srm, entry):
    """v / (1 + e^-v): the exponential loses an ulp (2^-23) and its product with v half of one, the sum half of one, the reciprocal one, the
    last product half of one: 3.5 2^-23.  A gate's product with y = 1 is exact, the state is one product with dt = 1 and one with B = silu(40),
    40 within half an ulp."""
    H = 4096
    v = torch.cat([torch.linspace(-80, 80, 3 * H), torch.linspace(-8, 8, H)]).float()
    if entry == "step bf16":
        v = v.to(BF16).float()
    got = []
    for k in range(0, v.numel(), H):
        part = v[None, k:k + H].cuda()
        out = torch.empty(1, H, device="cuda")
        if entry == "conv":
            srm.causal_conv(part, torch.ones(H, 1, device="cuda"), None, [0, 1], _i32([0, 1]), out)
            got.append(out.view(-1))
            continue
        dtype = BF16 if entry == "step bf16" else F32
        gate = entry.startswith("gate")
        dt, a, state = torch.ones(1, H, device="cuda"), torch.zeros(H, device="cuda"), torch.zeros(1, H, 1, 1, device="cuda")
        if gate:
            xbc = torch.zeros(1, H + 2, device="cuda")
            xbc[:, :H] = 1.0
            kw = dict(skip=torch.ones(H, device="cuda"), z=part, softplus=False, state=state)
            if entry == "gate of the scan":
                srm.selective_scan(xbc, dt, a, [0, 1], _i32([0, 1]), out, **kw)
            else:
                srm.selective_step(xbc, dt, a, _i32([0]), out=out, **kw)
            got.append(out.view(-1))
            continue
        xbc, bias = torch.zeros(1, H + 2, device="cuda"), torch.zeros(H + 2, device="cuda")
        xbc[:, :H], bias[H] = part, 40.0
        ring = torch.zeros(1, 1, H + 2, dtype=dtype, device="cuda")
        srm.selective_step(xbc.to(dtype), dt, a, _i32([0]), state, out.to(dtype), weight=torch.ones(H + 2, 1, device="cuda"), bias=bias, conv_state=ring,
                           softplus=False)
        got.append(state.view(-1) / 40.0)
    torch.cuda.synchronize()
    got, v = torch.cat(got).double().cpu(), v.double()
    want = v * recur_ref.sigmoid(v)
    wrong = torch.where(want == 0, 0.0, (got - want).abs() / want.abs().clamp_min(1e-300))
    print(f"{entry}: {float(wrong.max()):.2e} at {float(v[wrong.argmax()]):.4f}", flush=True)
    assert wrong.max() <= (3.5 + (2.0 if entry.startswith("step") else 0.0)) * 2.0 ** -23


@pytest.mark.parametrize("H,P,G,N", [(2, 4, 1, 1), (2, 70, 2, 3), (1, 64, 1, 5), (2, 20, 1, 13), (1, 40, 1, 27), (2, 50, 1, 37), (1, 64, 1, 100), (1, 33, 1, 200)])
@pytest.mark.parametrize("entry", ["scan", "step fp32", "step bf16"])
def test_an_infinite_x_is_an_infinity_in_y(srm, entry, H, P, G, N):
    """B and C above 0, no skip: the state of the channel and y are infinite from the token on, whatever lies behind the last of state_dim's
    lanes."""
    gen = torch.Generator().manual_seed(N)
    dtype, T = BF16 if entry == "step bf16" else F32, 40
    xbc = torch.randn(T, H * P + 2 * G * N, generator=gen)
    xbc[:, H * P:] = 0.5 + torch.rand(T, 2 * G * N, generator=gen)
    xbc[19, 2], xbc[7, H * P - 1] = math.inf, -math.inf
    xbc = xbc.to(dtype)
    dt, a = 0.1 + torch.rand(T, H, generator=gen), -torch.rand(H, generator=gen)
    state = torch.randn(1, H, P, N, generator=gen)
    want, size, after, mag = recur_ref.scan(xbc, dt, a, [0, T], H, P, G, N, softplus=False, pos=[3], state=state)
    out, held = torch.empty(T, H * P, dtype=dtype, device="cuda"), state.cuda()
    if entry == "scan":
        srm.selective_scan(xbc.cuda(), dt.cuda(), a.cuda(), [0, T], _i32([0, T]), out, groups=G, softplus=False, pos=_i32([3]), state=held)
    else:
        rows, sizes = xbc.cuda(), dt.cuda()
        for t in range(T):
            srm.selective_step(rows[t:t + 1], sizes[t:t + 1], a.cuda(), _i32([3 + t]), held, out[t:t + 1], groups=G, softplus=False)
    torch.cuda.synchronize()
    x = xbc[:, :H * P].double()
    want = torch.where(torch.isinf(x), x, want)                # (the reference multiplies by the skip that is not there)
    assert torch.isinf(want).sum() == 21 + 33 and not want.isnan().any()
    for got, ref, bound in ((out, want, recur_ref.scan_bounds(want, size, mag, T, N, dtype, False)[0]), (held, after, (2 * T + 64) * 2.0 ** -24 * mag)):
        got, far = got.double().cpu(), torch.isinf(ref)
        assert torch.equal(got[far], ref[far])
        assert ((got - ref).abs() <= bound)[~far].all()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("T,N", [(50, 64), (400, 64), (400, 37), (90, 128)])
def test_what_is_not_finite_in_b_or_c_stays_in_its_group_and_behind_its_token(srm, dtype, T, N):
    gen = torch.Generator().manual_seed(T + N)
    H, P, G = 4, 40, 2
    off, rows = [0, T, T + 40], T + 40
    xbc = torch.randn(rows, H * P + 2 * G * N, generator=gen).to(dtype).cuda()
    dt, a, z = torch.rand(rows, H, generator=gen).cuda(), -torch.rand(H, generator=gen).cuda(), torch.randn(rows, H * P, generator=gen).to(dtype).cuda()
    b_at, c_at = H * P, H * P + G * N

    def run(rows_of):
        out, state = torch.empty(rows, H * P, dtype=dtype, device="cuda"), torch.zeros(2, H, P, N, device="cuda")
        srm.selective_scan(rows_of, dt, a, off, _i32(off), out, groups=G, z=z, softplus=False, state=state)
        torch.cuda.synchronize()
        return out, state

    clean, held = run(xbc)
    for value in (math.inf, math.nan):
        bad = xbc.clone()
        bad[37, c_at + 5] = value                              # C of group 0: this token alone
        out, state = run(bad)
        touched = torch.zeros(rows, H * P, dtype=torch.bool, device="cuda")
        touched[37, :2 * P] = True
        assert torch.equal(out[~touched], clean[~touched]) and torch.equal(state, held)
        assert not torch.isfinite(out[touched]).any()
        bad = xbc.clone()
        bad[21, b_at + N + 3] = value                          # B of group 1: from this token on
        out, state = run(bad)
        touched[37] = False
        touched[21:T, 2 * P:] = True
        assert torch.equal(out[~touched], clean[~touched])
        assert not torch.isfinite(out[touched]).any()
        far = torch.zeros_like(state, dtype=torch.bool)
        far[0, 2:, :, 3] = True
        assert torch.equal(state[~far], held[~far]) and not torch.isfinite(state[far]).any()
