"""What the speed of the 8-bit operators and of sampling by request is measured on, through the public binding.

A case is one pass of one of four operators:

  norm      residual addition and root-mean-square norm, the normalised rows in 8 bits with scales
  quantize  rows of activations or weights to 8 bits with scales
  linear    the product of two such matrices, with the epilogues of the framework's linear layer
  sample    one token for each row of logits, with that row's temperature, top-k, top-p, min-p and random number

They follow each other at the end of a decode step (norm, head, tokens) and in a block (norm, up projection, quantize, down
projection into the residual stream).

An 8-bit matrix is `q` [rows][Kp], e4m3, Kp = K rounded up to 128 and zero behind K, and `scales` [ceil(K / 512)][rows][4], E8M0:
scales[b // 4, r, b % 4] belongs to q[r, 128 b : 128 b + 128].  A block's scale is the smallest power of two (2^-126 at least) that brings
its largest finite magnitude to 448 or less, 1 for a block of zeros and behind the last block.
"""
from __future__ import annotations

import math

import torch

own = False

E4M3, E8M0 = torch.float8_e4m3fn, torch.float8_e8m0fnu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}
STORE, GELU, RESIDUAL, LOGITS = 0, 1, 2, 4                              # epilogues of a linear layer
EPS = 1e-5


# ------------------------------------------------------------------ cases
def listed():
    return [
        # one user of the large benchmark model: a step of one row, where a launch's latency counts
        dict(name="norm_single", kind="norm", rows=1, d=1024, x="fp32", add="fp32", pad=0),
        # the large model's benchmark batch: fp32 residual stream, what a projection left in bf16 joins it
        dict(name="norm_large", kind="norm", rows=16384, d=1024, x="fp32", add="bf16", pad=0),
        # a few dozen users: the middle activations of the large model's MLP in front of its down projection
        dict(name="quantize_dozens", kind="quantize", rows=37, d=4096, x="bf16", pad=0),
        # an odd batch of odd rows that lie in a wider array
        dict(name="quantize_odd", kind="quantize", rows=3001, d=4001, x="bf16", pad=7),
        # one user: the head reads all of its 32000 rows for one row of logits
        dict(name="linear_single", kind="linear", M=1, N=32000, K=1024, epilogue=LOGITS, bias=False),
        # an odd few dozen users: the MLP's up projection with its activation
        dict(name="linear_dozens", kind="linear", M=37, N=4096, K=1024, epilogue=GELU, bias=True),
        # sizes that no tile divides, added into an fp32 residual stream
        dict(name="linear_odd", kind="linear", M=3001, N=4001, K=1000, epilogue=RESIDUAL, bias=True),
        # the down projection of the large benchmark batch, left in bf16 for the next norm to add
        dict(name="linear_down", kind="linear", M=16384, N=1024, K=4096, epilogue=STORE, bias=True),
        # a wide model's projection over a long prefill: the largest product
        dict(name="linear_large", kind="linear", M=8192, N=8192, K=8192, epilogue=STORE, bias=False),
        # one user: one row of logits, all filters on
        dict(name="sample_single", kind="sample", rows=1, vocab=32000, x="fp32", mode="mixed", pad=0),
        # a server's batch, every request with parameters of its own (greedy, plain, top-k, top-p, min-p, masks)
        dict(name="sample_batch", kind="sample", rows=300, vocab=32000, x="fp32", mode="mixed", pad=0),
        # rollouts with top-p from logits in bf16 over a large vocabulary of odd size
        dict(name="sample_large", kind="sample", rows=1000, vocab=128001, x="bf16", mode="top_p", pad=7),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, even in its logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    kind = rng.choice(["norm", "quantize", "linear", "linear", "sample", "sample"])
    x = rng.choice(["fp32", "bf16"])
    pad = rng.choice([0, 0, 8, rng.randrange(1, 64)])
    if kind in ("norm", "quantize"):
        d = _log(rng, 1, 16384)
        d = d if rng.random() < 0.4 else min(16384, -(-d // 64) * 64)
        rows = _log(rng, 1, min(65536, (1 << 25) // d))
        case = dict(kind=kind, rows=rows, d=d, x=x, pad=pad)
        if kind == "norm":
            case["add"] = rng.choice(["none", "fp32", "bf16"])
        return case
    if kind == "linear":
        K = _log(rng, 1, 8192)
        N = _log(rng, 1, 32768)
        M = _log(rng, 1, max(1, min(65536, (1 << 38) // (N * max(K, 128)), (1 << 28) // N)))
        if rng.random() < 0.6:
            K, N = -(-K // 128) * 128, -(-N // 16) * 16
        return dict(kind=kind, M=M, N=N, K=K, epilogue=rng.choice([STORE, GELU, RESIDUAL, LOGITS]), bias=rng.random() < 0.5)
    vocab = _log(rng, 1, 150000)
    rows = _log(rng, 1, min(4096, max(1, 100_000_000 // vocab)))
    return dict(kind=kind, rows=rows, vocab=vocab, x=x, mode=rng.choice(["plain", "top_k", "top_p", "mixed"]), pad=pad)


def _padded(d):
    return -(-d // 128) * 128


def _groups(d):
    return -(-d // 512)


def _size(name):
    return {"none": 0, "fp32": 4, "bf16": 2}[name]


def work(case):
    kind = case["kind"]
    if kind in ("norm", "quantize"):
        rows, d = case["rows"], case["d"]
        moved = rows * (_padded(d) + _groups(d) * 4) + rows * d * _size(case["x"])
        if kind == "quantize":
            return {"bytes": moved, "flops": 3 * rows * d}
        if case["add"] != "none":
            moved += rows * d * (_size(case["x"]) + _size(case["add"]))
        return {"bytes": moved + 4 * d, "flops": 8 * rows * d}
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        out = {STORE: 2, GELU: 2, RESIDUAL: 8, LOGITS: 4}[case["epilogue"]]
        return {"bytes": (M + N) * (_padded(K) + 4 * _groups(K)) + M * N * out + (4 * N if case["bias"] else 0), "flops": 2 * M * N * K}
    rows, vocab = case["rows"], case["vocab"]
    return {"bytes": rows * (vocab * _size(case["x"]) + 28), "flops": 4 * rows * vocab}


# ------------------------------------------------------------------ inputs
def _rows(gen, rows, d, pad, dtype, scale=1.0):
    """Normal rows with some columns ten times as large, as residual streams have them; `pad` columns more in memory."""
    wide = torch.randn((rows, d + pad), generator=gen, device="cuda") * scale
    wide[:, 3 % (d + pad)::97] *= 10.0
    return wide.to(dtype)[:, :d]


def _matrix(gen, rows, K, scale):
    x = torch.randn((rows, K), generator=gen, device="cuda") * scale
    return _to_fp8(x)


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    s = {"case": dict(case)}
    if kind in ("norm", "quantize"):
        rows, d = case["rows"], case["d"]
        s["x"] = _rows(gen, rows, d, case["pad"], TYPES[case["x"]])
        s["q"] = torch.empty((rows, _padded(d)), dtype=torch.uint8, device="cuda").view(E4M3)
        s["scales"] = torch.empty((_groups(d), rows, 4), dtype=torch.uint8, device="cuda").view(E8M0)
        if kind == "norm":
            s["gain"] = 1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")
            s["add"] = None if case["add"] == "none" else _rows(gen, rows, d, case["pad"], TYPES[case["add"]], 0.5)
        return s
    if kind == "linear":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"], s["a_scales"] = _matrix(gen, M, K, 1.0)
        s["w"], s["w_scales"] = _matrix(gen, N, K, 0.02)
        s["bias"] = 0.02 * torch.randn(N, generator=gen, device="cuda") if case["bias"] else None
        if case["epilogue"] == RESIDUAL:
            s["out"] = torch.randn((M, N), generator=gen, device="cuda")
        else:
            s["out"] = torch.empty((M, N), dtype=torch.float32 if case["epilogue"] == LOGITS else torch.bfloat16, device="cuda")
        return s
    rows, vocab, mode = case["rows"], case["vocab"], case["mode"]
    wide = torch.randn((rows, vocab + case["pad"]), generator=gen, device="cuda") * 2.5
    at = torch.randint(0, vocab, (rows, 8), generator=gen, device="cuda")
    wide.scatter_add_(1, at, 8.0 * torch.rand((rows, 8), generator=gen, device="cuda"))        # a few likely tokens
    wide = wide.to(TYPES[case["x"]])

    def one_of(values, dtype):
        pick = torch.randint(0, len(values), (rows,), generator=gen, device="cuda")
        return torch.tensor(values, dtype=dtype, device="cuda")[pick]

    s["temperature"] = one_of([0.6, 0.7, 1.0, 1.3] + ([0.0] if mode == "mixed" else []), torch.float32)
    s["top_k"] = one_of([1, 20, 50, 400] + ([0, 0, 0] if mode == "mixed" else []), torch.int32) if mode in ("top_k", "mixed") else None
    s["top_p"] = one_of([0.5, 0.9, 0.95] + ([1.0, 1.0] if mode == "mixed" else []), torch.float32) if mode in ("top_p", "mixed") else None
    s["min_p"] = one_of([0.0, 0.0, 0.02, 0.1], torch.float32) if mode == "mixed" else None
    s["uniform"] = torch.rand(rows, generator=gen, device="cuda")
    if mode == "mixed":                                                 # a grammar allows some requests a part of the vocabulary
        part = torch.rand((rows, 1), generator=gen, device="cuda")
        masked = (torch.rand((rows, vocab + case["pad"]), generator=gen, device="cuda") < 0.7) & (part < 0.2)
        wide.masked_fill_(masked, -math.inf)
    s["logits"] = wide[:, :vocab]
    s["tok"] = torch.empty(rows, dtype=torch.int32, device="cuda")
    s["logprob"] = torch.empty(rows, dtype=torch.float32, device="cuda")
    return s


# ------------------------------------------------------------------ one pass
def _to_fp8(y):
    """Plain form of the 8-bit format: y [rows][K] fp32 -> q, scales."""
    rows, K = y.shape
    blocks = torch.nn.functional.pad(y, (0, _groups(K) * 512 - K)).view(rows, -1, 128)
    finite = torch.isfinite(blocks)
    largest = torch.where(finite, blocks.abs(), 0.0).amax(-1)
    mantissa, exponent = torch.frexp(largest)                           # largest = mantissa 2^exponent, mantissa in [0.5, 1)
    exponent = (exponent - 9 + (mantissa > 0.875)).clamp_min(-126)      # 448 = 0.875 * 2^9
    exponent = torch.where(largest == 0, 0, exponent)
    q = torch.where(finite, torch.ldexp(blocks, -exponent[..., None]), math.nan).to(E4M3).view(rows, -1)[:, :_padded(K)].contiguous()
    scales = (exponent + 127).to(torch.uint8).view(rows, -1, 4).transpose(0, 1).contiguous().view(E8M0)
    return q, scales


def _from_fp8(q, scales, dtype=torch.float32):
    rows, Kp = q.shape
    by_block = scales.view(torch.uint8).transpose(0, 1).reshape(rows, -1)[:, : Kp // 128]
    factor = torch.exp2(by_block.to(dtype) - 127.0)
    return (q.to(dtype).view(rows, -1, 128) * factor[..., None]).view(rows, Kp)


def _plain_norm(s):
    x = s["x"]
    if s["add"] is not None:
        x.copy_(x.float() + s["add"].float())
    v = x.float()
    y = v * torch.rsqrt(v.square().mean(-1, keepdim=True) + EPS) * s["gain"]
    return (x, *_to_fp8(y))


def _plain_linear(s):
    v = _from_fp8(s["a"], s["a_scales"]) @ _from_fp8(s["w"], s["w_scales"]).t()
    if s["bias"] is not None:
        v = v + s["bias"]
    epilogue, out = s["case"]["epilogue"], s["out"]
    if epilogue == RESIDUAL:
        return out.add_(v)
    if epilogue == GELU:
        v = 0.5 * v * (1.0 + torch.erf(v * math.sqrt(0.5)))
    return out.copy_(v)


def _plain_sample(s):
    """In 64 bits, as a sum's rounding next to a border would choose another token."""
    x = s["logits"].double()
    rows, V = x.shape
    x = torch.where(x.isnan(), -math.inf, x)
    top = x.amax(-1, keepdim=True)
    t = s["temperature"].double()[:, None]
    greedy = ~(t > 0)
    weight = torch.where(x == top, 1.0, torch.exp((x - top) / torch.where(greedy, 1.0, t)))
    weight = torch.where(x == -math.inf, 0.0, weight)
    order = torch.sort(x, dim=-1, descending=True, stable=True).indices
    sorted_w = weight.gather(1, order)
    rank = torch.arange(V, device=x.device)[None, :]
    limit = torch.where(greedy, 1, V)
    if s["top_k"] is not None:
        k = s["top_k"].long()[:, None]
        limit = torch.where((k > 0) & ~greedy, k, limit)
    kept = rank < limit
    if s["min_p"] is not None:
        least = s["min_p"].double()[:, None]
        kept &= ~((least > 0) & (sorted_w < least.clamp_max(1.0)))
    if s["top_p"] is not None:
        p = s["top_p"].double()[:, None]
        left = torch.where(kept, sorted_w, 0.0)
        before = left.cumsum(-1) - left
        kept &= ~(p < 1) | (before < p * left.sum(-1, keepdim=True)) | (rank == 0)
    mass = torch.zeros_like(weight).scatter_(1, order, torch.where(kept, sorted_w, 0.0))
    upto = mass.cumsum(-1)
    total = upto[:, -1:]
    u = s["uniform"].double()[:, None]
    tok = (upto <= u * total).sum(-1)
    last = torch.where(mass > 0, rank, -1).amax(-1)                     # -1: nothing to choose from
    tok = torch.minimum(tok, last)
    logprob = torch.log(mass.gather(1, tok.clamp_min(0)[:, None]) / total)[:, 0]
    logprob = torch.where(tok < 0, -math.inf, logprob)
    return s["tok"].copy_(tok), s["logprob"].copy_(logprob)


def run(s):
    kind = s["case"]["kind"]
    if own:
        import paper_2605_08696_amd as srm
        if kind == "norm":
            srm.rmsnorm_fp8(s["x"], s["gain"], EPS, s["q"], s["scales"], add=s["add"])
            return s["x"], s["q"], s["scales"]
        if kind == "quantize":
            srm.quantize_fp8(s["x"], s["q"], s["scales"])
            return s["q"], s["scales"]
        if kind == "linear":
            srm.linear_fp8(s["case"]["epilogue"], s["a"], s["a_scales"], s["w"], s["w_scales"], s["bias"], s["out"])
            return s["out"]
        srm.sample_rows(s["logits"], s["uniform"], s["tok"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                        min_p=s["min_p"], logprob=s["logprob"])
        return s["tok"], s["logprob"]
    if kind == "norm":
        return _plain_norm(s)
    if kind == "quantize":
        return _to_fp8(s["x"].float())
    if kind == "linear":
        return _plain_linear(s)
    return _plain_sample(s)


# ------------------------------------------------------------------ the definition, in 64 bits
def _exact_fp8(y):
    """The values that the format keeps of y (64 bits), and its scales: nearest multiples of the step at each magnitude, ties to even."""
    rows, K = y.shape
    held = torch.zeros((rows, _groups(K) * 4, 128), dtype=torch.float64, device=y.device)
    held.view(rows, -1)[:, :K] = y
    peak = held.abs().amax(-1, keepdim=True)
    scale = torch.exp2(torch.ceil(torch.log2(peak / 448.0)))
    scale = torch.where(peak > 448.0 * scale, 2.0 * scale, scale)       # where the logarithm was rounded across a power of two
    scale = torch.where(peak <= 224.0 * scale, 0.5 * scale, scale).clamp_min(2.0 ** -126)
    scale = torch.where(peak == 0, 1.0, scale)
    v = held / scale
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp_min(2.0 ** -6))) - 3)
    q = torch.round(v / step) * step
    return q.view(rows, -1)[:, : _padded(K)].contiguous(), scale.view(rows, -1, 4).permute(1, 0, 2).contiguous()


def _exact_sample(s):
    logits = s["logits"]
    found = torch.full((logits.shape[0],), -math.inf, dtype=torch.float64, device=logits.device)
    host = {k: None if s[k] is None else s[k].tolist() for k in ("temperature", "top_k", "top_p", "min_p", "uniform")}
    for r in range(logits.shape[0]):
        x = logits[r].double()
        V, most, t = x.numel(), x.max(), host["temperature"][r]
        if most == -math.inf:
            continue
        if not t > 0:
            found[r] = 0.0
            continue
        # highest first; of equal logits the stable sort of the negated row keeps the lowest index in front
        value, index = torch.sort(-x, stable=True)
        w = torch.exp((-value - most) / t)
        n = V
        if host["top_k"] and host["top_k"][r] > 0:
            n = min(n, host["top_k"][r])
        if host["min_p"] and host["min_p"][r] > 0:
            n = min(n, int(torch.count_nonzero(w >= min(host["min_p"][r], 1.0))))
        if host["top_p"] and host["top_p"][r] < 1:
            sums = torch.cumsum(w[:n], 0)
            n = 1 + int(torch.count_nonzero(sums[:-1] < host["top_p"][r] * sums[-1]))
        index, back = torch.sort(index[:n])
        w = w[:n][back]
        sums = torch.cumsum(w, 0)
        at = min(int(torch.searchsorted(sums, host["uniform"][r] * sums[-1], right=True)), n - 1)
        found[r] = torch.log(w[at]) - torch.log(sums[-1])
    return found


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "quantize":
        return _exact_fp8(s["x"].double())
    if kind == "norm":
        x = s["x"].double()
        if s["add"] is not None:
            x = x + s["add"].double()
        kept = x.to(TYPES[case["x"]]).double()                          # the norm is that of the rows as they are stored
        norm = torch.sqrt((kept * kept).sum(-1, keepdim=True) / case["d"] + EPS)
        return (x, *_exact_fp8(kept / norm * s["gain"].double()))
    if kind == "linear":
        Kp = s["a"].shape[1]

        def values(q, scales):
            by_block = scales.float().double().permute(1, 0, 2).reshape(q.shape[0], -1)[:, : Kp // 128]
            return q.double() * torch.repeat_interleave(by_block, 128, dim=1)

        v = torch.matmul(values(s["a"], s["a_scales"]), values(s["w"], s["w_scales"]).t().contiguous())
        if s["bias"] is not None:
            v += s["bias"].double()
        if case["epilogue"] == GELU:
            v = v * torch.special.ndtr(v)
        return s["out"].double() + v if case["epilogue"] == RESIDUAL else v
    return None, _exact_sample(s)
