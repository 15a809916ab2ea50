"""The selective recurrence, its short convolution and scores of tokens in 64 bits, token by token (torch, on the CPU).

Beside each result stands its size: the same sums of magnitudes, which the bounds of rounding errors are multiples of."""
import math

import torch

F64 = torch.float64


def sigmoid(v):
    return torch.where(v >= 0, 1 / (1 + torch.exp(-v.clamp_min(0))), torch.exp(v.clamp_max(0)) / (1 + torch.exp(v.clamp_max(0))))


def conv(x, weight, bias, offsets, pos, slot, state, activation=True):
    """(out, v in front of the activation, size of v, state): out has zeros where a sequence is idle and NaN outside all of them."""
    x, weight = x.to(F64), weight.to(F64)
    W, slots = weight.shape[1], 0 if state is None else state.shape[0]
    bias = torch.zeros(x.shape[1], dtype=F64) if bias is None else bias.to(F64)
    out = torch.full_like(x, math.nan)
    v, size = out.clone(), out.clone()
    after = None if state is None else state.to(F64).clone()
    for n, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        kept = state[slot[n]].to(F64) if 0 <= slot[n] < slots else None
        if pos[n] < 0:
            out[lo:hi], v[lo:hi], size[lo:hi] = 0.0, 0.0, 0.0
            continue
        for t in range(lo, hi):
            acc, mag = bias.clone(), bias.abs()
            for k in range(W):
                at = t - (W - 1) + k
                p = pos[n] + at - lo
                row = x[at] if at >= lo else kept[p % W] if p >= 0 and kept is not None else torch.zeros_like(x[0])
                acc += weight[:, k] * row
                mag += weight[:, k].abs() * row.abs()
            v[t], size[t] = acc, mag
            out[t] = acc * sigmoid(acc) if activation else acc
        if kept is not None:
            for t in range(max(lo, hi - W), hi):
                after[slot[n], (pos[n] + t - lo) % W] = x[t]
    return out, v, size, after


def conv_bound(out, v, size, W, dtype, activation=True):
    """W products and W sums in fp32; the activation's slope is below 1.1, its exponential's argument is rounded (|v| 2^-24), its exponential,
    sum, reciprocal and product lose 2^-23 each; one rounding to the output's type."""
    fp32 = (W + 1) * 2.0 ** -24 * size * 1.01
    if activation:
        fp32 = 1.1 * fp32 + (v.abs() + 4) * 2.0 ** -23 * out.abs()
    return fp32 + torch.finfo(dtype).eps / 2 * 1.01 * out.abs() + 1e-37


def split(rows, H, P, G, N):
    x, b, c = torch.split(rows.to(F64), [H * P, G * N, G * N], dim=-1)
    of = torch.arange(H) // (H // G)
    return x.unflatten(-1, (H, P)), b.unflatten(-1, (G, N))[..., of, :], c.unflatten(-1, (G, N))[..., of, :]


def sizes(dt, dt_bias, softplus):
    dt = dt.to(F64) + (0 if dt_bias is None else dt_bias.to(F64))
    return dt.clamp_min(0) + torch.log1p(torch.exp(-dt.abs())) if softplus else dt


def scan(xbc, dt, a, offsets, H, P, G, N, dt_bias=None, skip=None, z=None, softplus=True, pos=None, slot=None, state=None):
    """(out, size of out, state, size of state, tokens that reach into each sequence's state)."""
    rows = xbc.shape[0]
    x, b, c = split(xbc, H, P, G, N)
    dt, a = sizes(dt, dt_bias, softplus), a.to(F64)
    skip = torch.zeros(H, dtype=F64) if skip is None else skip.to(F64)
    n_seq, slots = len(offsets) - 1, 0 if state is None else state.shape[0]
    pos = [0] * n_seq if pos is None else pos
    slot = list(range(n_seq)) if slot is None else slot
    out, size = (torch.full((rows, H * P), math.nan, dtype=F64) for _ in range(2))
    after = None if state is None else state.to(F64).clone()
    mag = None if state is None else after.abs()
    for n, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        if pos[n] < 0:
            out[lo:hi], size[lo:hi] = 0.0, 0.0
            continue
        kept = 0 <= slot[n] < slots
        S = state[slot[n]].to(F64).clone() if kept and pos[n] > 0 else torch.zeros(H, P, N, dtype=F64)
        M = S.abs()
        for t in range(lo, hi):
            decay = torch.exp(dt[t] * a)[:, None, None]
            S = decay * S + (dt[t][:, None] * x[t])[..., None] * b[t][:, None, :]
            M = decay * M + (dt[t].abs()[:, None] * x[t].abs())[..., None] * b[t].abs()[:, None, :]
            y = (S * c[t][:, None, :]).sum(-1) + skip[:, None] * x[t]
            m = (M * c[t].abs()[:, None, :]).sum(-1) + skip.abs()[:, None] * x[t].abs()
            out[t], size[t] = y.flatten(), m.flatten()
        if kept and hi > lo:
            after[slot[n]], mag[slot[n]] = S, M
    if z is not None:
        gate = z.to(F64)
        gate = gate * sigmoid(gate)
        out, size = out * gate, size * gate.abs()
    return out, size, after, mag


def scan_bounds(out, size, mag, T, N, dtype, matrix, gate=None):
    """(of out, of the state).  fp32: an element of the state is a sum of at most T terms, two roundings a step, each term's decay off by its
    exponents' roundings (their sum E counts 2^-E E <= 0.54 at 2^-21 of dt's and the products' roundings) and dt, x, B by 2^-20 together; y is
    N products and sums more.  On the matrix cores one more rounding to bf16 (2^-8) of what is multiplied by C, or by x.  Then the gate
    (|z| up to 8: 12 2^-23) and the output's rounding."""
    state = (2 * T + 64) * 2.0 ** -24 * mag + 1e-30
    y = (2 * T + N + 96) * 2.0 ** -24 * size + (2.0 ** -8 * 1.01 * size if matrix else 0.0)
    return y + (torch.finfo(dtype).eps / 2 * 1.01) * out.abs() + 1e-30, state


def score(l, token=None, top=0, temperature=1.0):
    """(log p of the token, entropy, top tokens, their log p) of one row, by sorting."""
    l = l.to(F64)
    l = torch.where(l.isnan(), -math.inf, l)
    V, m = l.numel(), l.max().item()
    t = min(max(temperature, 1e-30), 1e30) if temperature > 0 else 1.0
    if m == -math.inf:
        logs = torch.full_like(l, -math.inf)
    elif m == math.inf:
        logs = torch.where(l == math.inf, -math.log(int((l == math.inf).sum())), -math.inf)
    else:
        d = (l - m) / t
        logs = d - torch.log(torch.exp(d).sum())
    p = torch.exp(logs)
    entropy = -(p[p > 0] * logs[p > 0]).sum().item()
    order = torch.sort(-l, stable=True).indices[:top]
    order = [int(i) for i in order if l[i] > -math.inf]
    given = 0.0 if token is None or not 0 <= token < V else logs[token].item()
    return given, entropy, order + [-1] * (top - len(order)), [logs[i].item() for i in order] + [-math.inf] * (top - len(order))
