"""The operators that need no model beside what a model makes: the MLP of a layer in 8 bits behind srm_mixer_block, tokens by request
from a decode step's logits; and their kernels' first launches under capture."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

import fp8_ref
import srm_synth
from gpu_util import to_dev

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _values(q, s):
    exp = fp8_ref.scale_exponents(s.view(torch.uint8).cpu().numpy(), q.shape[1] // 128)
    return torch.from_numpy(fp8_ref.dequantize(q.double().cpu().numpy(), exp)).cuda()


def _check_quantized(x, q, s):
    want, exp = fp8_ref.quantize(x.double().cpu().numpy())
    np.testing.assert_array_equal(s.view(torch.uint8).cpu().numpy(), fp8_ref.scale_words(exp))
    np.testing.assert_array_equal(q.double().cpu().numpy(), want)


@pytest.mark.parametrize("d,B", [(256, 1), (256, 37), (512, 333)])
def test_the_mlp_of_a_layer_in_8_bits(srm, d, B):
    """mixer_block leaves LayerNorm2's rows; quantize, up projection with GELU, quantize, down projection into the residual stream.  Each
    step against 64 bits on what the step before has left.  A product loses 2^-23 of the magnitudes' sum in each of K + 3 steps, one
    with a bf16 output 7 * 2^-13 of it besides and 2^-8 of its value; the GELU's slope is below 1.13, its fitted form 6.5e-7 off."""
    cfg = srm_synth.tiny_config(vocab=16, d_model=d, n_layers=2, n_heads=4, n_ctx=8, weight_dtype="bf16", seed=81)
    w = srm_synth.make_weights(cfg)
    model = srm.Model(cfg, w)
    ff, lw = cfg.d_ff, w["layers"][1]
    rng = np.random.default_rng(B)
    x = to_dev((rng.standard_normal((B, d)) * 1.5).astype(np.float32))
    S = to_dev(rng.standard_normal((B, d)).astype(np.float32))
    norm = torch.empty(B, d, dtype=torch.bfloat16, device="cuda")
    up, down = srm.fp8_empty(ff, d), srm.fp8_empty(d, ff)
    srm.quantize_fp8(to_dev(lw["w_up"]), *up)
    srm.quantize_fp8(to_dev(lw["w_down"]), *down)
    b_up, b_down = to_dev(lw["b_up"]), to_dev(lw["b_down"])
    q, qh = srm.fp8_empty(B, d), srm.fp8_empty(B, ff)
    h = torch.empty(B, ff, dtype=torch.bfloat16, device="cuda")

    model.mixer_block(1, 6, B, x, S, norm)
    before = x.double()
    srm.quantize_fp8(norm, *q)
    srm.linear_fp8(1, *q, *up, b_up, h)
    srm.quantize_fp8(h, *qh)
    srm.linear_fp8(2, *qh, *down, b_down, x)
    torch.cuda.synchronize()
    _check_quantized(norm, *q)
    _check_quantized(to_dev(lw["w_up"]), *up)
    _check_quantized(h, *qh)
    v = _values(*q) @ _values(*up).t().contiguous() + b_up.double()
    size = _values(*q).abs() @ _values(*up).abs().t().contiguous() + b_up.double().abs()
    want = v * torch.special.ndtr(v)
    assert ((h.double() - want).abs() <= 1.13 * ((d + 3) * 2.0 ** -23 + 7 * 2.0 ** -13) * size + 1e-6 + 2.0 ** -8 * 1.01 * want.abs()).all()
    v = before + _values(*qh) @ _values(*down).t().contiguous() + b_down.double()
    size = before.abs() + _values(*qh).abs() @ _values(*down).abs().t().contiguous() + b_down.double().abs()
    assert ((x.double() - v).abs() <= (ff + 3) * 2.0 ** -23 * size).all()
    model.close()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_tokens_by_request_from_a_decode_steps_logits(srm, dtype):
    """A generation in which each request has parameters of its own: the tokens are those of the rule in 64 bits from the step's logits,
    those of greedy requests the step's own."""
    cfg = srm_synth.tiny_config(vocab=1031, d_model=256, n_layers=2, n_heads=4, n_ctx=32, weight_dtype=dtype, seed=82)
    model = srm.Model(cfg, srm_synth.make_weights(cfg, stress=True))
    B, P, G = 23, 5, 6
    rng = np.random.default_rng(7)
    prompts = to_dev(rng.integers(0, cfg.vocab, (B, P)).astype(np.int32))
    state, ws = model.new_state(B), model.new_workspace(B * P)
    logits = torch.empty(B, cfg.vocab, device="cuda")
    own, tok = torch.empty(B, dtype=torch.int32, device="cuda"), torch.empty(B, dtype=torch.int32, device="cuda")
    logprob = torch.empty(B, device="cuda")
    host = dict(temperature=rng.choice([0.0, 0.5, 1.0, 1.5], B), top_k=rng.choice([0, 5, 40], B), top_p=rng.choice([0.5, 0.9, 1.0], B),
                min_p=rng.choice([0.0, 0.02], B))
    host = {k: v.astype(np.int32 if k == "top_k" else np.float32) for k, v in host.items()}
    cols = {k: to_dev(v) for k, v in host.items()}
    greedy = host["temperature"] == 0
    assert greedy.any() and not greedy.all()
    model.prefill(prompts, 1, state, own, logits=logits, workspace=ws)
    for g in range(G):
        u = rng.random(B).astype(np.float32)
        srm.sample_rows(logits, to_dev(u), tok, logprob=logprob, **cols)
        got, lp, rows = tok.cpu().numpy(), logprob.double().cpu().numpy(), logits.double().cpu().numpy()
        for r in range(B):
            want, logp, near = fp8_ref.sample(rows[r], u=float(u[r]), temperature=float(host["temperature"][r]), top_k=int(host["top_k"][r]),
                                              top_p=float(host["top_p"][r]), min_p=float(host["min_p"][r]))
            assert near > 1e-11 and got[r] == want, (g, r)
            assert abs(lp[r] - logp) <= 2.0 ** -24 * abs(logp) * 1.01 + 1e-9, (g, r)
        np.testing.assert_array_equal(got[greedy], own.cpu().numpy()[greedy])
        model.decode_step(B, P + g, tok, state, own, logits=logits, workspace=ws)
    torch.cuda.synchronize()
    model.close()


FIRST_LAUNCHES = """
import torch
import paper_2605_08696_amd as srm

srm.lib()
M, d, ff, N = 300, 1024, 2048, 4096
x, gain = torch.zeros(M, d, device="cuda"), torch.ones(d, device="cuda")
q, qh = srm.fp8_empty(M, d), srm.fp8_empty(M, ff)
weights = [(torch.randint(0, 0x40, (n, k), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn),
            torch.full(((k + 511) // 512, n, 4), 120, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu))
           for n, k in ((ff, d), (N, ff), (N, 256))]
h = torch.empty(M, ff, dtype=torch.bfloat16, device="cuda")
logits, u, tok = torch.empty(M, N, device="cuda"), torch.rand(M, device="cuda"), torch.empty(M, dtype=torch.int32, device="cuda")
large = torch.empty(N, N, dtype=torch.bfloat16, device="cuda")
small, tall = torch.empty(5, ff, dtype=torch.bfloat16, device="cuda"), torch.empty(3001, 2060, device="cuda")
qt = [t[:3001] for t in weights[2][:1]] + [weights[2][1][:, :3001].contiguous()]
wt = [weights[2][0][:2060], weights[2][1][:, :2060].contiguous()]
q5 = srm.fp8_empty(5, d)


def run():
    srm.rmsnorm_fp8(x, gain, 1e-5, *q)
    srm.linear_fp8(1, *q, *weights[0], None, h)
    srm.quantize_fp8(h, *qh)
    srm.linear_fp8(4, *qh, *weights[1], None, logits)
    srm.sample_rows(logits, u, tok)
    srm.quantize_fp8(x[:5], *q5)
    srm.linear_fp8(0, *q5, *weights[0], None, small)                # K cut over the wavefronts
    srm.linear_fp8(0, *weights[2], *weights[2], None, large)        # the persistent kernel, all of a CU's LDS
    srm.linear_fp8(4, *qt, *wt, None, tall)                         # tiles


torch.cuda.synchronize()
graph = torch.cuda.CUDAGraph()
with torch.cuda.graph(graph):
    run()
kept = (q[0], q[1], h, qh[0], qh[1], logits, tok, small, large, tall)
for i in range(4):
    x.normal_()
    graph.replay()
    torch.cuda.synchronize()
    replayed = [t.view(torch.uint8).clone() for t in kept]
    for t in kept:
        t.view(torch.uint8).zero_()
    run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(replayed, kept)), i
    assert tok.unique().numel() > 1 and large.float().amax() > 0
print("replays equal")
"""


def test_first_launches_under_capture():
    """In a process of its own, whose first launch of every kernel is captured: each replay has the bits of the eager calls."""
    out = subprocess.run([sys.executable, "-c", FIRST_LAUNCHES], cwd=ROOT, env={**os.environ, "PYTHONPATH": ROOT}, capture_output=True, text=True,
                         timeout=100)
    assert out.returncode == 0 and "replays equal" in out.stdout, out.stdout + out.stderr
