"""The selective recurrence, its convolution and the scores of tokens as they are used: behind each other and beside what the framework has,
captured and replayed, on other streams, two at once."""
import numpy as np
import pytest
import torch

import recur_ref
import srm_synth
from gpu_util import to_dev

pytestmark = pytest.mark.gpu
BF16 = torch.bfloat16


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


class Layer:
    """A layer's weights, and its states in `slots` slots."""

    def __init__(self, seed, H, P, G, N, W, slots, dtype):
        gen = torch.Generator().manual_seed(seed)
        self.H, self.P, self.G, self.N, self.W, self.C, self.dtype = H, P, G, N, W, H * P + 2 * G * N, dtype
        self.weight, self.bias = (torch.randn(self.C, W, generator=gen) * 0.5).cuda(), (torch.randn(self.C, generator=gen) * 0.1).cuda()
        self.a, self.dt_bias, self.skip = -torch.exp(torch.randn(H, generator=gen)).cuda(), torch.randn(H, generator=gen).cuda() - 2, torch.randn(H, generator=gen).cuda()
        self.state = torch.full((slots, H, P, N), float("nan"), device="cuda")       # what a slot held before does not matter
        self.ring = torch.full((slots, W, self.C), float("nan"), dtype=dtype, device="cuda")

    def prompts(self, srm, rows, dt, z, offsets, d_offsets, conv, out, pos, slot, stream=None):
        srm.causal_conv(rows, self.weight, self.bias, offsets, d_offsets, conv, pos=pos, slot=slot, state=self.ring, stream=stream)
        srm.selective_scan(conv, dt, self.a, offsets, d_offsets, out, groups=self.G, dt_bias=self.dt_bias, skip=self.skip, z=z, pos=pos, slot=slot,
                           state=self.state, stream=stream)

    def step(self, srm, rows, dt, z, pos, slot, out, stream=None):
        srm.selective_step(rows, dt, self.a, pos, self.state, out, groups=self.G, weight=self.weight, bias=self.bias, conv_state=self.ring,
                           dt_bias=self.dt_bias, skip=self.skip, z=z, slot=slot, stream=stream)


def _rows(gen, n, layer):
    w = lambda cols: torch.randn(n, cols, generator=gen).to(layer.dtype).cuda()  # noqa: E731
    return w(layer.C), w(layer.H), w(layer.H * layer.P)


@pytest.mark.parametrize("dtype", [torch.float32, BF16])
def test_prompts_in_parts_then_tokens_are_the_whole_sequence(srm, dtype):
    """A conversation's prompt in two calls among others', then tokens one at a time, gives what one call over all of it gives: against the
    whole in 64 bits (from what the convolution has left of each token, rounded to dtype or not; so twice the rounding's bound)."""
    gen = torch.Generator().manual_seed(1)
    layer = Layer(2, 4, 64, 2, 64, 4, 5, dtype)
    lengths, slots, more = [130, 1, 47], [3, 0, 4], 9
    rows, dt, z = zip(*[_rows(gen, n + more, layer) for n in lengths])
    got = [torch.empty(n + more, layer.H * layer.P, dtype=dtype, device="cuda") for n in lengths]
    done = [0, 0, 0]
    for part in ([100, 0, 2], [30, 1, 45]):
        off = np.concatenate([[0], np.cumsum(part)]).astype(np.int32)
        pick = lambda t: torch.cat([t[i][done[i]:done[i] + part[i]] for i in range(3)])  # noqa: E731
        x, d, g = pick(rows), pick(dt), pick(z)
        conv, out = torch.empty_like(x), torch.empty_like(g)
        layer.prompts(srm, x, d, g, off, _i32(off.tolist()), conv, out, _i32(done), _i32(slots))
        for i in range(3):
            got[i][done[i]:done[i] + part[i]] = out[off[i]:off[i + 1]]
            done[i] += part[i]
    for k in range(more):
        at = [n + k for n in lengths]
        x, d, g = (torch.stack([t[i][at[i]] for i in range(3)]) for t in (rows, dt, z))
        out = torch.empty_like(g)
        layer.step(srm, x, d, g, _i32(at), _i32(slots), out)
        for i in range(3):
            got[i][at[i]] = out[i]
    torch.cuda.synchronize()
    for i in range(3):
        n = lengths[i] + more
        conv, v, size, _ = recur_ref.conv(rows[i].cpu(), layer.weight.cpu(), layer.bias.cpu(), [0, n], [0], [-1], None)
        wrong = recur_ref.conv_bound(conv, v, size, layer.W, dtype)
        kw = dict(dt=dt[i].cpu(), a=layer.a.cpu(), offsets=[0, n], H=layer.H, P=layer.P, G=layer.G, N=layer.N, dt_bias=layer.dt_bias.cpu(), skip=layer.skip.cpu(),
                  z=z[i].cpu())
        want, mag, _, _ = recur_ref.scan(conv, **kw)
        _, up, _, _ = recur_ref.scan(conv.abs() + wrong, **kw)
        bound, _ = recur_ref.scan_bounds(want, mag, mag, n, layer.N, dtype, dtype is BF16)
        # (x, B and C wrong by `wrong` at most, all in the direction of their size; the bound of the scan's own roundings, on the larger sums)
        over = (got[i].double().cpu() - want).abs() - 1.01 * (up - mag) - 1.05 * bound
        assert (over <= 0).all(), (i, float(over.max()))


def test_a_scan_layer_in_8_bits_to_scored_tokens(srm):
    """Prompts through convolution, scan, norm and head in 8 bits, and the scores of their own next tokens: each step against 64 bits on
    what the step before has left."""
    gen = torch.Generator().manual_seed(4)
    layer = Layer(5, 8, 64, 1, 128, 4, 4, BF16)
    V, off = 1031, [0, 33, 90, 91]
    T, d = off[-1], layer.H * layer.P
    rows, dt, z = _rows(gen, T, layer)
    conv, out = torch.empty_like(rows), torch.empty_like(z)
    layer.prompts(srm, rows, dt, z, np.array(off, dtype=np.int32), _i32(off), conv, out, None, None)
    gain, w = torch.ones(d, device="cuda"), torch.randn(V, d, generator=gen).cuda()
    q, wq = srm.fp8_empty(T, d), srm.fp8_empty(V, d)
    srm.quantize_fp8(w, *wq)
    srm.rmsnorm_fp8(out, gain, 1e-5, *q)
    logits = torch.empty(T, V, device="cuda")
    srm.linear_fp8(4, *q, *wq, None, logits)
    token = torch.randint(0, V, (T,), generator=gen).to(torch.int32)
    token[[32, 89, 90]] = -1                                   # the prompts' last rows have no next token
    lp, en = torch.empty(T, device="cuda"), torch.empty(T, device="cuda")
    tt, tl = torch.empty(T, 5, dtype=torch.int32, device="cuda"), torch.empty(T, 5, device="cuda")
    srm.token_logprobs(logits, token.cuda(), lp, entropy=en, top_token=tt, top_logprob=tl)
    torch.cuda.synchronize()
    want, v, size, _ = recur_ref.conv(rows.cpu(), layer.weight.cpu(), layer.bias.cpu(), off, [0, 0, 0], [-1, -1, -1], None)
    assert ((conv.double().cpu() - want).abs() <= recur_ref.conv_bound(want, v, size, layer.W, BF16)).all()
    want, mag, _, _ = recur_ref.scan(conv.cpu(), dt.cpu(), layer.a.cpu(), off, layer.H, layer.P, layer.G, layer.N, dt_bias=layer.dt_bias.cpu(),
                                     skip=layer.skip.cpu(), z=z.cpu())
    bound, _ = recur_ref.scan_bounds(want, mag, mag, 57, layer.N, BF16, True)
    assert ((out.double().cpu() - want).abs() <= bound).all()
    host = logits.double().cpu()
    for r in range(T):
        given, entropy, tokens, logs = recur_ref.score(host[r], int(token[r]), 5)
        assert tt[r].tolist() == tokens
        assert abs(lp[r].item() - given) <= 2e-5 and abs(en[r].item() - entropy) <= 2e-5      # (logits up to some 60: 2^-24 of |d| + log Z, and Z)
        assert np.abs(tl[r].cpu().numpy() - logs).max() <= 2e-5
    assert (lp[[32, 89, 90]] == 0).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scores_of_a_models_own_logits(srm, dtype):
    """The prompt's tokens scored from parallel_forward's logits; a decode step's greedy token is the first of its top tokens."""
    cfg = srm_synth.tiny_config(vocab=1031, d_model=256, n_layers=2, n_heads=4, n_ctx=32, weight_dtype=dtype, seed=82)
    model = srm.Model(cfg, srm_synth.make_weights(cfg, stress=True))
    B, T = 3, 17
    rng = np.random.default_rng(7)
    prompts = to_dev(rng.integers(0, cfg.vocab, (B, T)).astype(np.int32))
    hidden, logits, ws = torch.empty(B, T, cfg.d_model, device="cuda"), torch.empty(B, T, cfg.vocab, device="cuda"), model.new_workspace(B * T)
    model.parallel_forward(prompts, hidden, logits, ws)
    given = torch.cat([prompts[:, 1:], torch.full((B, 1), -1, dtype=torch.int32, device="cuda")], 1).contiguous()
    lp = torch.empty(B * T, device="cuda")
    srm.token_logprobs(logits.view(B * T, -1), given.view(-1), lp)
    state, tok = model.new_state(B), torch.empty(B, dtype=torch.int32, device="cuda")
    step_logits = torch.empty(B, cfg.vocab, device="cuda")
    model.decode_step(B, 0, prompts[:, 0].contiguous(), state, tok, logits=step_logits, workspace=ws)
    top, top_lp = torch.empty(B, 3, dtype=torch.int32, device="cuda"), torch.empty(B, 3, device="cuda")
    srm.token_logprobs(step_logits, None, None, top_token=top, top_logprob=top_lp)
    torch.cuda.synchronize()
    assert torch.equal(top[:, 0], tok)
    want = torch.log_softmax(logits.double(), -1).gather(2, given.clamp_min(0).long()[..., None])[..., 0]
    want[:, -1] = 0.0
    assert ((lp.view(B, T).double() - want).abs() <= 1e-6 * (1 + want.abs())).all()
    model.close()


def test_captured_and_replayed_with_other_inputs(srm):
    """Scan of two prompts (one cut into segments), step and scores in one graph, replayed over new inputs in the same buffers, with eager work
    and synchronizations between: each replay gives the eager call's bits."""
    gen = torch.Generator().manual_seed(6)
    layer, other = (Layer(7, 2, 64, 1, 128, 4, 2, BF16) for _ in range(2))
    off = np.array([0, 700, 733], dtype=np.int32)
    T, d_off = int(off[-1]), _i32(off.tolist())
    assert srm.selective_scan_workspace_bytes(srm.SRM_BF16, off, 2, 64, 128) > 0
    rows, dt, z = _rows(gen, T, layer)
    conv, out = torch.empty_like(rows), torch.empty_like(z)
    pos, slot, pos1 = _i32([0, 0]), _i32([1, 0]), _i32([700, 33])
    step_out = torch.empty(2, layer.H * layer.P, dtype=BF16, device="cuda")
    logits, token = torch.randn(2, 40001, generator=gen).cuda(), _i32([5, 7])
    lp, tt, tl = torch.empty(2, device="cuda"), torch.empty(2, 20, dtype=torch.int32, device="cuda"), torch.empty(2, 20, device="cuda")

    def work(layer, stream=None):
        layer.prompts(srm, rows, dt, z, off, d_off, conv, out, pos, slot, stream)
        layer.step(srm, rows[:2], dt[:2], z[:2], pos1, _i32_slot, step_out, stream)
        srm.token_logprobs(logits, token, lp, top_token=tt, top_logprob=tl, stream=stream)

    _i32_slot = slot
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):                              # (the kernels' first launches are captured ones)
        work(layer)
    for k in range(4):
        r, d, g = _rows(gen, T, layer)
        rows.copy_(r), dt.copy_(d), z.copy_(g), logits.copy_(torch.randn(2, 40001, generator=gen))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (conv, out, step_out, lp, tt, tl, layer.state, layer.ring)]
        work(other)
        torch.cuda.synchronize()
        for a, b in zip(got, (conv, out, step_out, lp, tt, tl, other.state, other.ring)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), k


def test_two_at_once_on_streams_of_their_own(srm):
    """Two scans with workspaces allocated in the call, and steps behind them, on two streams: the bits of the same one after the other."""
    gen = torch.Generator().manual_seed(9)
    off = np.array([0, 2000], dtype=np.int32)
    d_off = _i32(off.tolist())
    slot = _i32([0])
    runs = []
    for seed in (1, 2):
        rows, dt, z = _rows(gen, 2000, Layer(seed, 2, 64, 1, 64, 4, 1, BF16))
        runs.append([Layer(seed, 2, 64, 1, 64, 4, 1, BF16), Layer(seed, 2, 64, 1, 64, 4, 1, BF16), rows, dt, z])
    pos = _i32([2000])
    outs = [[torch.empty_like(r[4]) for _ in range(2)] + [torch.empty_like(r[2]) for _ in range(2)] for r in runs]
    steps = [[torch.empty_like(r[4][:1]) for _ in range(2)] for r in runs]
    for i, r in enumerate(runs):
        r[0].prompts(srm, r[2], r[3], r[4], off, d_off, outs[i][2], outs[i][0], None, slot)
        r[0].step(srm, r[2][:1], r[3][:1], r[4][:1], pos, slot, steps[i][0])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in runs]
    for i, (r, st) in enumerate(zip(runs, streams)):
        r[1].prompts(srm, r[2], r[3], r[4], off, d_off, outs[i][3], outs[i][1], None, slot, stream=st)
        r[1].step(srm, r[2][:1], r[3][:1], r[4][:1], pos, slot, steps[i][1], stream=st)
    torch.cuda.synchronize()
    for i, r in enumerate(runs):
        assert torch.equal(outs[i][0], outs[i][1]) and torch.equal(steps[i][0], steps[i][1]) and torch.equal(r[0].state, r[1].state)


def test_a_call_gives_the_same_bits_again(srm):
    """Sums have one order: twice the same call, with and without the others of its batch."""
    gen = torch.Generator().manual_seed(11)
    layer = Layer(3, 4, 64, 1, 128, 4, 3, BF16)
    lengths = [200, 64, 77]
    off = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int32)
    rows, dt, z = _rows(gen, int(off[-1]), layer)
    got = []
    for _ in range(2):
        conv, out = torch.empty_like(rows), torch.empty_like(z)
        layer.prompts(srm, rows, dt, z, off, _i32(off.tolist()), conv, out, None, None)
        torch.cuda.synchronize()
        got.append((out, layer.state.clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    one = torch.empty(64, layer.H * layer.P, dtype=BF16, device="cuda")
    state = torch.empty(1, layer.H, layer.P, layer.N, device="cuda")
    srm.selective_scan(conv[200:264], dt[200:264], layer.a, [0, 64], _i32([0, 64]), one, dt_bias=layer.dt_bias, skip=layer.skip, z=z[200:264], state=state)
    torch.cuda.synchronize()
    assert torch.equal(one, out[200:264]) and torch.equal(state[0], layer.state[1])
