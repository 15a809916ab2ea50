"""What the speed of the selective recurrence and of scored tokens is measured on, through the public binding.

A case is one pass of one of four operators:

  conv     the short causal convolution of packed prompts, every channel by itself, with SiLU
  scan     the selective recurrence over packed prompts: a matrix of state for each head, whose decay and input depend on the token
  step     both for one token of each request, in place in the requests' slots
  score    log probabilities of given tokens, with the entropy of each row of logits and its most likely tokens

A prompt goes through conv and scan to logits, whose tokens are scored; requests go on with step.

Rows of the recurrence are x [H][P] | B [G][N] | C [G][N].  With dt = softplus(dt_raw + dt_bias[h]) and g = h // (H / G):
  S[h, p, n] <- exp(dt A[h]) S[h, p, n] + dt x[h, p] B[g, n]      y[h, p] = sum_n S[h, p, n] C[g, n] + D[h] x[h, p]      out = y silu(z)
A slot keeps S in fp32 and the last `width` rows before the convolution, position p in row p % width.  At position 0 both count as zeros.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
BLOCK = 64                                                              # tokens of a block of the plain form


# ------------------------------------------------------------------ cases
def listed():
    return [
        # a few dozen new tokens of one conversation of the large benchmark model's width, in front of a scan
        dict(name="conv_chunk", kind="conv", prompts=1, tokens=37, channels=2304, width=4, x="bf16", first=False, pad=0),
        # a long prefill of several requests of a wide model
        dict(name="conv_large", kind="conv", prompts=8, tokens=32768, channels=4352, width=4, x="bf16", first=True, pad=0),
        # one user's short prompt in a small model, where launches count
        dict(name="scan_short", kind="scan", prompts=1, tokens=37, heads=16, dim=64, groups=1, state=64, x="bf16", dt="bf16", z=True, first=True, pad=0),
        # a server's prompts of all lengths, later parts of conversations among them
        dict(name="scan_ragged", kind="scan", prompts=37, tokens=11111, heads=32, dim=64, groups=1, state=128, x="bf16", dt="bf16", z=True, first=False, pad=0),
        # one long document: little but time to split
        dict(name="scan_long", kind="scan", prompts=1, tokens=16384, heads=32, dim=64, groups=1, state=128, x="bf16", dt="fp32", z=False, first=True, pad=0),
        # sizes that no tile divides, in fp32, rows that lie in a wider array
        dict(name="scan_odd", kind="scan", prompts=5, tokens=1667, heads=10, dim=50, groups=2, state=37, x="fp32", dt="fp32", z=True, first=False, pad=5),
        # a long prefill of several requests of a wide model: the largest scan
        dict(name="scan_large", kind="scan", prompts=8, tokens=32768, heads=64, dim=64, groups=8, state=128, x="bf16", dt="bf16", z=True, first=True, pad=0),
        # one user: the next token
        dict(name="step_single", kind="step", rows=1, heads=32, dim=64, groups=1, state=128, width=4, x="bf16", dt="bf16", z=True, pad=0),
        # a server's batch: every request's matrices of state are read and written
        dict(name="step_batch", kind="step", rows=300, heads=32, dim=64, groups=1, state=128, width=4, x="bf16", dt="bf16", z=True, pad=0),
        # one user: the token that was chosen, with the alternatives that are shown beside it
        dict(name="score_single", kind="score", rows=1, vocab=32000, x="fp32", top=20, temperature=False, pad=0),
        # the tokens of a prompt of 500, from the large benchmark model's logits
        dict(name="score_prompt", kind="score", rows=500, vocab=32000, x="fp32", top=5, temperature=False, pad=0),
        # rollouts that are scored at their own temperatures, from logits in bf16 over a large vocabulary of odd size
        dict(name="score_large", kind="score", rows=2001, vocab=128001, x="bf16", top=20, temperature=True, pad=7),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even in its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def _heads(rng):
    groups = rng.choice([1, 1, 1, 2, 4, 8])
    heads = groups * _log(rng, 1, 64 // groups)
    dim = rng.choice([16, 32, 64, 64, 64, 128, rng.randrange(1, 129)])
    state = rng.choice([16, 32, 64, 128, 128, 256, rng.randrange(1, 257)])
    return dict(heads=heads, dim=dim, groups=groups, state=state)


def draw(rng):
    kind = rng.choice(["conv", "scan", "scan", "scan", "step", "step", "score", "score"])
    x = rng.choice(["bf16", "bf16", "fp32"])
    pad = rng.choice([0, 0, 8, rng.randrange(1, 64)])
    if kind == "conv":
        channels = _log(rng, 1, 8192)
        channels = channels if rng.random() < 0.3 else -(-channels // 64) * 64
        tokens = _log(rng, 1, min(65536, (32768 * 2176) // channels))
        return dict(kind=kind, prompts=_log(rng, 1, min(tokens, 300)), tokens=tokens, channels=channels, width=rng.choice([2, 3, 4, 4, 4, 8]), x=x,
                    first=rng.random() < 0.5, pad=pad)
    if kind == "score":
        vocab = _log(rng, 1, 150000)
        rows = _log(rng, 1, min(4096, max(1, 100_000_000 // vocab)))
        return dict(kind=kind, rows=rows, vocab=vocab, x=x, top=rng.choice([0, 1, 5, 20, 32]), temperature=rng.random() < 0.5, pad=pad)
    sizes = _heads(rng)
    dt = rng.choice([x, x, "fp32"])
    per_token = sizes["heads"] * sizes["dim"] * sizes["state"]
    if kind == "step":
        return dict(kind=kind, rows=_log(rng, 1, min(1024, max(1, (1 << 27) // per_token))), width=rng.choice([2, 3, 4, 4, 4]), x=x, dt=dt,
                    z=rng.random() < 0.7, pad=pad, **sizes)
    tokens = _log(rng, 1, max(1, min(20000, (1 << 33) // per_token, (1 << 23) // sizes["heads"])))
    return dict(kind=kind, prompts=_log(rng, 1, min(tokens, 64)), tokens=tokens, x=x, dt=dt, z=rng.random() < 0.7, first=rng.random() < 0.5, pad=pad, **sizes)


def _size(name):
    return {"fp32": 4, "bf16": 2}[name]


def work(case):
    kind, size = case["kind"], _size(case["x"])
    if kind == "conv":
        T, C, W = case["tokens"], case["channels"], case["width"]
        return {"bytes": 2 * T * C * size + (1 if case["first"] else 2) * case["prompts"] * W * C * size + 4 * C * (W + 1), "flops": (2 * W + 5) * T * C}
    if kind == "score":
        rows, V = case["rows"], case["vocab"]
        return {"bytes": rows * (V * size + 12 + 8 * case["top"] + (4 if case["temperature"] else 0)), "flops": 6 * rows * V}
    H, P, G, N = case["heads"], case["dim"], case["groups"], case["state"]
    rows = case["rows"] if kind == "step" else case["tokens"]
    moved = rows * ((H * P * (3 if case["z"] else 2) + 2 * G * N) * size + H * _size(case["dt"])) + 12 * H
    held = 4 * H * P * N
    if kind == "step":
        ring = (case["width"] + 1) * (H * P + 2 * G * N) * size
        return {"bytes": moved + rows * (2 * held + ring), "flops": 6 * rows * H * P * N}
    return {"bytes": moved + case["prompts"] * held * (1 if case["first"] else 2), "flops": 6 * rows * H * P * N}


# ------------------------------------------------------------------ inputs
def _lengths(gen, prompts, tokens):
    """Offsets of `prompts` prompts of one token at least, `tokens` in all; equal ones where they divide, as benchmarks have them."""
    if tokens % prompts == 0 and tokens // prompts >= 1024:
        return torch.arange(prompts + 1, dtype=torch.int32) * (tokens // prompts)
    share = 0.05 + torch.rand(prompts, generator=gen, device="cuda").double().cpu()
    ends = torch.floor(torch.cumsum(share, 0) / share.sum() * (tokens - prompts)).long()
    ends[-1] = tokens - prompts
    ends += torch.arange(1, prompts + 1)
    return torch.cat([torch.zeros(1, dtype=torch.long), ends]).to(torch.int32)


def _slots(gen, n):
    """A slot for each of n requests, among a few more."""
    return torch.randperm(n + 3, generator=gen, device="cuda")[:n].to(torch.int32)


def _wide(gen, rows, cols, pad, dtype):
    return torch.randn((rows, cols + pad), generator=gen, device="cuda").to(dtype)[:, :cols]


# (A state's values are sums of dt x B over some 1 / (dt |A|) tokens, about 0.02.)
def _prepare_heads(gen, case, rows, s):
    H, P, G, N = case["heads"], case["dim"], case["groups"], case["state"]
    x = TYPES[case["x"]]
    # step sizes of 0.001 to 0.1, even in their logarithm, moved by the token; decays of 1 to 16 a unit of time
    size = torch.exp(math.log(0.001) + math.log(100.0) * torch.rand(H, generator=gen, device="cuda"))
    s["dt_bias"] = size + torch.log(-torch.expm1(-size))
    s["dt"] = _wide(gen, rows, H, case["pad"], TYPES[case["dt"]])
    s["a"] = -(1.0 + 15.0 * torch.rand(H, generator=gen, device="cuda"))
    s["skip"] = 1.0 + 0.1 * torch.randn(H, generator=gen, device="cuda")
    s["z"] = _wide(gen, rows, H * P, case["pad"], x) if case["z"] else None
    s["out"] = torch.zeros((rows, H * P + case["pad"]), dtype=x, device="cuda")[:, : H * P]
    s["channels"] = H * P + 2 * G * N


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, x = case["kind"], TYPES[case["x"]]
    s = {"case": dict(case)}
    if kind == "score":
        rows, V = case["rows"], case["vocab"]
        wide = torch.randn((rows, V + case["pad"]), generator=gen, device="cuda") * 2.5
        at = torch.randint(0, V, (rows, 8), generator=gen, device="cuda")
        wide.scatter_add_(1, at, 8.0 * torch.rand((rows, 8), generator=gen, device="cuda"))    # a few likely tokens
        s["logits"] = wide.to(x)[:, :V]
        # most given tokens are likely ones, some any, and a few rows have none (the ends of padded requests)
        part = torch.rand(rows, generator=gen, device="cuda")
        token = torch.where(part < 0.7, at[:, 0], torch.randint(0, V, (rows,), generator=gen, device="cuda"))
        s["token"] = torch.where(part > 0.97, -1, token).to(torch.int32)
        s["temperature"] = 0.6 + 0.8 * torch.rand(rows, generator=gen, device="cuda") if case["temperature"] else None
        s["logprob"], s["entropy"] = (torch.empty(rows, device="cuda") for _ in range(2))
        s["top_token"] = torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda") if case["top"] else None
        s["top_logprob"] = torch.empty((rows, case["top"]), device="cuda") if case["top"] else None
        return s
    if kind == "step":
        rows, W = case["rows"], case["width"]
        _prepare_heads(gen, case, rows, s)
        s["pos"] = torch.randint(0, 4000, (rows,), generator=gen, device="cuda").to(torch.int32)
        s["slot"] = _slots(gen, rows)
        s["x"] = _wide(gen, rows, s["channels"], case["pad"], x)
        s["ring"] = torch.randn((rows + 3, W, s["channels"]), generator=gen, device="cuda").to(x)
        s["weight"] = torch.randn((s["channels"], W), generator=gen, device="cuda") / math.sqrt(W)
        s["bias"] = 0.1 * torch.randn(s["channels"], generator=gen, device="cuda")
        s["state"] = torch.randn((rows + 3, case["heads"], case["dim"], case["state"]), generator=gen, device="cuda") * 0.02
        return s
    prompts, T = case["prompts"], case["tokens"]
    s["offsets"] = _lengths(gen, prompts, T)
    s["d_offsets"] = s["offsets"].cuda()
    s["slot"] = _slots(gen, prompts)
    s["pos"] = torch.randint(0, 4000, (prompts,), generator=gen, device="cuda").to(torch.int32)
    if case["first"]:
        s["pos"].zero_()
    else:
        s["pos"][::3] = 0                                               # new conversations among old ones
        s["pos"][:1] = 777
    if kind == "conv":
        C, W = case["channels"], case["width"]
        s["x"] = _wide(gen, T, C, case["pad"], x)
        s["weight"] = torch.randn((C, W), generator=gen, device="cuda") / math.sqrt(W)
        s["bias"] = 0.1 * torch.randn(C, generator=gen, device="cuda")
        s["ring"] = torch.randn((prompts + 3, W, C), generator=gen, device="cuda").to(x)
        s["out"] = torch.zeros((T, C + case["pad"]), dtype=x, device="cuda")[:, :C]
        return s
    _prepare_heads(gen, case, T, s)
    v = torch.randn((T, s["channels"] + case["pad"]), generator=gen, device="cuda")
    s["x"] = (v / (1.0 + torch.exp(-v))).to(x)[:, : s["channels"]]      # as the convolution leaves rows
    s["state"] = torch.randn((prompts + 3, case["heads"], case["dim"], case["state"]), generator=gen, device="cuda") * 0.02
    return s


# ------------------------------------------------------------------ one pass: the plain form
def _silu(v):
    return v / (1.0 + torch.exp(-v))


def _softplus(v):
    return v.clamp_min(0.0) + torch.log1p(torch.exp(-v.abs()))


def _tokens(s):
    """For each token of the packed prompts: its prompt and its position."""
    off = s["d_offsets"].long()
    of = torch.repeat_interleave(torch.arange(off.numel() - 1, device=off.device), off.diff())
    return of, s["pos"].long()[of] + torch.arange(of.numel(), device=off.device) - off[of]


def _plain_conv(s):
    x, ring, off = s["x"], s["ring"], s["d_offsets"].long()
    T, C = x.shape
    W = s["case"]["width"]
    of, at = _tokens(s)
    back = torch.arange(W - 1, -1, -1, device=x.device)
    token, position = torch.arange(T, device=x.device)[:, None] - back, at[:, None] - back
    kept = T + s["slot"].long()[of][:, None] * W + position % W         # where what came before the call's tokens lies
    source = torch.cat([x, ring.view(-1, C), x.new_zeros(1, C)])
    row = torch.where(position < 0, source.shape[0] - 1, torch.where(token >= off[of][:, None], token, kept))
    v = (source[row].float() * s["weight"].t()).sum(1) + s["bias"]
    s["out"].copy_(_silu(v))
    end = s["pos"].long() + off.diff()
    last = end[:, None] - 1 - (end[:, None] - 1 - torch.arange(W, device=x.device)) % W        # the position that each row of a ring holds
    new = last >= s["pos"].long()[:, None]
    row = torch.where(new, off[:-1, None] + last - s["pos"].long()[:, None], 0)
    slot = s["slot"].long()
    ring[slot] = torch.where(new[..., None], x[row], ring[slot])
    return s["out"], ring


def _plain_scan(s):
    case, off = s["case"], s["d_offsets"].long()
    H, P, G, N = case["heads"], case["dim"], case["groups"], case["state"]
    lengths = off.diff()
    blocks = -(-int(s["offsets"].diff().max()) // BLOCK)
    S, T = lengths.numel(), s["x"].shape[0]
    at = torch.arange(blocks * BLOCK, device=off.device)
    there = at[None, :] < lengths[:, None]                              # prompts side by side, with empty tokens behind their ends
    row = torch.where(there, off[:-1, None] + at, 0)
    rows = torch.where(there[..., None], s["x"].float()[row], 0.0).view(S, blocks, BLOCK, -1)
    x = rows[..., : H * P].reshape(S, blocks, BLOCK, H, P).transpose(2, 3)                     # [S][blocks][H][BLOCK][P]
    b, c = (rows[..., H * P + i * G * N: H * P + (i + 1) * G * N].reshape(S, blocks, BLOCK, G, N).transpose(2, 3) for i in (0, 1))
    dt = _softplus(s["dt"].float() + s["dt_bias"])[row]
    dt = torch.where(there[..., None], dt, 0.0).view(S, blocks, BLOCK, H).transpose(2, 3)      # [S][blocks][H][BLOCK]
    upto = torch.cumsum(dt.double() * s["a"].double()[:, None], -1)
    part = upto[..., :, None] - upto[..., None, :]
    earlier = torch.arange(BLOCK, device=off.device)[:, None] >= torch.arange(BLOCK, device=off.device)
    decay = torch.exp(torch.where(earlier, part, -math.inf)).float()
    del part
    near = torch.repeat_interleave(c @ b.transpose(-1, -2).contiguous(), H // G, dim=2)
    y = (near * decay * dt[..., None, :]) @ x.contiguous()
    del near, decay
    weight = (torch.exp(upto[..., -1:] - upto) * dt).float()
    added = (x * weight[..., None]).transpose(-1, -2).contiguous() @ torch.repeat_interleave(b, H // G, dim=2)     # [S][blocks][H][P][N]
    # the state in front of every block, and behind the last: decayed sums of what the blocks before it and the slot bring
    start = torch.where((s["pos"] > 0)[:, None, None, None], s["state"][s["slot"].long()], 0.0)
    brought = torch.cat([start[:, None], added], 1).transpose(1, 2).reshape(S, H, blocks + 1, P * N)
    sums = torch.nn.functional.pad(torch.cumsum(upto[..., -1], 1), (0, 0, 1, 0)).transpose(1, 2)                   # [S][H][blocks + 1]
    part = sums[..., :, None] - sums[..., None, :]
    before = torch.arange(blocks + 1, device=off.device)[:, None] >= torch.arange(blocks + 1, device=off.device)
    carried = torch.exp(torch.where(before, part, -math.inf)).float() @ brought
    carried = carried.view(S, H, blocks + 1, P, N).transpose(1, 2)
    y += (torch.repeat_interleave(c, H // G, dim=2) @ carried[:, :-1].transpose(-1, -2).contiguous()) * torch.exp(upto).float()[..., None]
    y += s["skip"][:, None, None] * x
    y = y.transpose(2, 3).reshape(S, -1, H * P)[there]
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    s["out"].copy_(y)
    s["state"][s["slot"].long()] = carried[:, -1]
    return s["out"], s["state"]


def _plain_step(s):
    case = s["case"]
    H, P, G, N, W = case["heads"], case["dim"], case["groups"], case["state"], case["width"]
    rows, slot, pos = case["rows"], s["slot"].long(), s["pos"].long()
    s["ring"][slot, pos % W] = s["x"]
    position = pos[:, None] - torch.arange(W - 1, -1, -1, device=pos.device)
    taps = torch.where((position >= 0)[..., None], s["ring"][slot[:, None], position % W].float(), 0.0)
    v = _silu((taps * s["weight"].t()).sum(1) + s["bias"])
    x = v[:, : H * P].reshape(rows, H, P)
    b, c = (torch.repeat_interleave(v[:, H * P + i * G * N: H * P + (i + 1) * G * N].reshape(rows, G, N), H // G, dim=1) for i in (0, 1))
    dt = _softplus(s["dt"].float() + s["dt_bias"])
    held = torch.where((pos > 0)[:, None, None, None], s["state"][slot], 0.0)
    held = held * torch.exp(dt * s["a"])[..., None, None] + (dt[..., None] * x)[..., None] * b[:, :, None, :]
    s["state"][slot] = held
    y = (held * c[:, :, None, :]).sum(-1) + s["skip"][:, None] * x
    y = y.reshape(rows, -1)
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    s["out"].copy_(y)
    return s["out"], s["ring"], s["state"]


def _plain_score(s):
    x = s["logits"].float()
    rows, V = x.shape
    k = s["case"]["top"]
    x = torch.where(x.isnan(), -math.inf, x)
    v = x if s["temperature"] is None else x / s["temperature"][:, None]
    v = v - v.amax(-1, keepdim=True)
    weight = torch.exp(v)
    total = weight.sum(-1, keepdim=True)
    logs = v - torch.log(total)
    s["entropy"].copy_(-torch.where(weight > 0, weight * logs, 0.0).sum(-1) / total[:, 0])
    token = s["token"].long()
    given = (token >= 0) & (token < V)
    s["logprob"].copy_(torch.where(given, logs.gather(1, token.clamp(0, V - 1)[:, None])[:, 0], 0.0))
    if not k:
        return s["logprob"], s["entropy"]
    # whole numbers in the order of the logits, lower indexes first among equal ones
    bits = (x + 0.0).view(torch.int32).long()
    key = torch.where(bits < 0, bits ^ 0x7FFFFFFF, bits) * (1 << 31) - torch.arange(V, device=x.device)
    best = torch.topk(key, min(k, V), dim=-1).indices
    value = logs.gather(1, best)
    best = torch.where(value == -math.inf, -1, best)
    s["top_token"].fill_(-1)[:, : best.shape[1]] = best
    s["top_logprob"].fill_(-math.inf)[:, : best.shape[1]] = value
    return s["logprob"], s["entropy"], s["top_token"], s["top_logprob"]


def run(s):
    case = s["case"]
    kind = case["kind"]
    if own:
        import paper_2605_08696_amd as srm
        if kind == "conv":
            srm.causal_conv(s["x"], s["weight"], s["bias"], s["offsets"], s["d_offsets"], s["out"], pos=s["pos"], slot=s["slot"], state=s["ring"])
            return s["out"], s["ring"]
        if kind == "scan":
            srm.selective_scan(s["x"], s["dt"], s["a"], s["offsets"], s["d_offsets"], s["out"], groups=case["groups"], dt_bias=s["dt_bias"], skip=s["skip"],
                               z=s["z"], pos=s["pos"], slot=s["slot"], state=s["state"])
            return s["out"], s["state"]
        if kind == "step":
            srm.selective_step(s["x"], s["dt"], s["a"], s["pos"], s["state"], s["out"], groups=case["groups"], weight=s["weight"], bias=s["bias"],
                               conv_state=s["ring"], dt_bias=s["dt_bias"], skip=s["skip"], z=s["z"], slot=s["slot"])
            return s["out"], s["ring"], s["state"]
        srm.token_logprobs(s["logits"], s["token"], s["logprob"], temperature=s["temperature"], entropy=s["entropy"], top_token=s["top_token"],
                           top_logprob=s["top_logprob"])
        return (s["logprob"], s["entropy"]) + ((s["top_token"], s["top_logprob"]) if case["top"] else ())
    return {"conv": _plain_conv, "scan": _plain_scan, "step": _plain_step, "score": _plain_score}[kind](s)


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_conv(s):
    x, ring, out = s["x"].double(), s["ring"].double(), s["out"].double()
    kept, W = ring.clone(), s["case"]["width"]
    offsets, pos, slot = s["offsets"].tolist(), s["pos"].tolist(), s["slot"].tolist()
    for n, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        past = [ring[slot[n], p % W] if p >= 0 else torch.zeros_like(x[0]) for p in range(pos[n] - W + 1, pos[n])]
        line = torch.cat([torch.stack(past), x[lo:hi]]) if past else x[lo:hi]
        v = torch.nn.functional.conv1d(line.t()[None], s["weight"].double()[:, None, :], s["bias"].double(), groups=x.shape[1])[0].t()
        out[lo:hi] = v * torch.sigmoid(v)
        for t in range(max(lo, hi - W), hi):
            kept[slot[n], (pos[n] + t - lo) % W] = x[t]
    return out, kept


def _exact_step_of(s, held, x, b, c, dt, h_of):
    """One token: the state after it, and y."""
    held = held * torch.exp(dt * s["a"].double())[..., None, None] + torch.einsum("rh,rhp,rhn->rhpn", dt, x, b[:, h_of])
    return held, torch.einsum("rhpn,rhn->rhp", held, c[:, h_of]) + s["skip"].double()[:, None] * x


def _parts(s, rows):
    case = s["case"]
    H, P, G, N = case["heads"], case["dim"], case["groups"], case["state"]
    x, b, c = torch.split(rows, [H * P, G * N, G * N], dim=-1)
    return x.unflatten(-1, (H, P)), b.unflatten(-1, (G, N)), c.unflatten(-1, (G, N))


def _exact_gate(s, y, rows):
    if s["z"] is None:
        return y
    z = s["z"].double()[rows]
    return y * z * torch.sigmoid(z)


def _exact_scan(s):
    case = s["case"]
    h_of = torch.arange(case["heads"], device="cuda") // (case["heads"] // case["groups"])
    dt = torch.logaddexp(s["dt"].double() + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    offsets, slot = s["offsets"].long(), s["slot"].long()
    lengths = offsets.diff()
    order = torch.argsort(lengths, descending=True)                     # the prompts that still run are the first ones
    many = (lengths[order][None, :] > torch.arange(int(lengths.max()))[:, None]).sum(1).tolist()
    first, order = offsets[:-1][order].cuda(), order.cuda()
    held = torch.where((s["pos"] > 0)[:, None, None, None], s["state"][slot].double(), 0.0)[order]
    out, after = s["out"].double(), s["state"].double()
    for t, n in enumerate(many):
        rows = first[:n] + t
        x, b, c = _parts(s, s["x"][rows].double())
        held[:n], y = _exact_step_of(s, held[:n], x, b, c, dt[rows], h_of)
        out[rows] = y.flatten(1)
    after[slot[order]] = held
    return _exact_gate(s, out, slice(None)), after


def _exact_step(s):
    case = s["case"]
    h_of = torch.arange(case["heads"], device="cuda") // (case["heads"] // case["groups"])
    W, slot, pos = case["width"], s["slot"].long(), s["pos"].long()
    ring, after = s["ring"].double(), s["state"].double()
    v = s["bias"].double() + s["weight"].double()[:, W - 1] * s["x"].double()
    for back in range(1, W):
        v += torch.where((pos >= back)[:, None], ring[slot, (pos - back) % W], 0.0) * s["weight"].double()[:, W - 1 - back]
    ring[slot, pos % W] = s["x"].double()
    x, b, c = _parts(s, v * torch.sigmoid(v))
    dt = torch.logaddexp(s["dt"].double() + s["dt_bias"].double(), torch.zeros((), dtype=torch.float64, device="cuda"))
    held = torch.where((pos > 0)[:, None, None, None], after[slot], 0.0)
    held, y = _exact_step_of(s, held, x, b, c, dt, h_of)
    after[slot] = held
    return _exact_gate(s, y.flatten(1), slice(None)), ring, after


def _exact_score(s):
    logits, k = s["logits"], s["case"]["top"]
    rows, V = logits.shape
    logprob = torch.zeros(rows, dtype=torch.float64, device="cuda")
    entropy = torch.zeros_like(logprob)
    top = torch.full((rows, k), -math.inf, dtype=torch.float64, device="cuda")
    given = s["token"].tolist()
    temperature = None if s["temperature"] is None else s["temperature"].tolist()
    for r in range(rows):
        l = logits[r].double()
        if temperature:
            l = l / temperature[r]
        logs = torch.log_softmax(l, 0)
        entropy[r] = torch.special.entr(torch.exp(logs)).sum()
        if 0 <= given[r] < V:
            logprob[r] = logs[given[r]]
        n = min(k, V)
        if n:
            top[r, :n] = torch.topk(logs, n).values
    return (logprob, entropy) + ((None, top) if k else ())


def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "step": _exact_step, "score": _exact_score}[case["kind"]](s)
