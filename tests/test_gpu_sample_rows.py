"""Sampling by request through the public binding, against the rule in 64 bits (numpy).

Tokens have to be equal.  A draw that lies within 1e-11 of a border between two tokens, or a top-p target within 1e-11 of a running sum,
could go either way (weights are held to 2^-43 of the largest): the inputs are seeded, and no row comes that near, which is asserted unless
a test says strict=False (rows of equal or few values; test_gpu_sample_rows_ties.py has the rule in whole numbers for those).  A log probability is a difference of two numbers of 64 bits, rounded to fp32: 2^-24 relative, and 1e-9 for the sums."""
import math

import numpy as np
import pytest
import torch

import fp8_ref

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _column(values, dtype):
    return None if values is None else torch.tensor(np.asarray(values), dtype=dtype, device="cuda")


def check(srm, logits, u, temperature=None, top_k=None, top_p=None, min_p=None, strict=True):
    rows = logits.shape[0]
    tok = torch.full((rows + 2,), -7, dtype=torch.int32, device="cuda")
    lp = torch.full((rows + 2,), 7.0, device="cuda")
    f = torch.float32
    cols = dict(temperature=_column(temperature, f), top_k=_column(top_k, torch.int32), top_p=_column(top_p, f), min_p=_column(min_p, f))
    u = _column(u, f)
    print(f"sample_rows {logits.dtype} {rows} x {logits.shape[1]}, stride {logits.stride(0)}", flush=True)
    srm.sample_rows(logits, u, tok[1:-1], logprob=lp[1:-1], **cols)
    torch.cuda.synchronize()
    assert tok[0] == -7 and tok[-1] == -7 and lp[0] == 7 and lp[-1] == 7
    again = torch.empty(rows, dtype=torch.int32, device="cuda")
    srm.sample_rows(logits, u, again, **cols)                 # without log probabilities
    assert torch.equal(again, tok[1:-1])
    host = logits.double().cpu().numpy()
    col = {k: None if v is None else v.double().cpu().numpy() for k, v in cols.items()}
    uh = u.double().cpu().numpy()
    got_t, got_l = tok[1:-1].cpu().numpy(), lp[1:-1].double().cpu().numpy()
    for r in range(rows):
        kw = {k: v[r] for k, v in col.items() if v is not None}
        if "top_k" in kw:
            kw["top_k"] = int(kw["top_k"])
        want, logp, near = fp8_ref.sample(host[r], u=uh[r], **kw)
        assert not strict or near > 1e-11, (r, near)
        assert got_t[r] == want, (r, kw, uh[r], got_t[r], want)
        if math.isinf(logp):
            assert got_l[r] == logp
        else:
            assert abs(got_l[r] - logp) <= 2.0 ** -24 * abs(logp) * 1.01 + 1e-9, (r, got_l[r], logp)
    return got_t


def _logits(rng, rows, V, pad=0, dtype=torch.float32, offset=0, scale=3.0):
    flat = torch.zeros(offset + rows * (V + pad), dtype=dtype, device="cuda")
    t = flat[offset:].view(rows, V + pad)
    t.copy_(torch.from_numpy((rng.standard_normal((rows, V + pad)) * scale).astype(np.float32)))
    return t[:, :V]


VOCABS = [(1, 0, 0), (2, 1, 0), (7, 0, 1), (8, 3, 0), (9, 0, 0), (63, 0, 1), (64, 3, 0), (511, 0, 0), (512, 1, 1), (513, 0, 0), (1000, 5, 3), (1023, 0, 0), (1024, 2, 0), (1025, 0, 1), (4096, 0, 0), (8192, 0, 0), (8193, 0, 1), (32000, 0, 0),
          (32001, 8, 0), (50021, 1, 2), (131072, 0, 0), (150001, 0, 1)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,offset", VOCABS)
def test_parameters_of_every_kind_in_one_batch(srm, V, pad, offset, dtype):
    rng = np.random.default_rng(V)
    rows = 24 if V < 50000 else 10
    logits = _logits(rng, rows, V, pad, dtype, offset)
    check(srm, logits, rng.random(rows), temperature=rng.choice([0.0, 0.3, 0.7, 1.0, 2.0], rows), top_k=rng.choice([0, 1, 2, 20, 300, V, V + 5], rows),
          top_p=rng.choice([0.05, 0.5, 0.9, 0.99, 1.0], rows), min_p=rng.choice([0.0, 0.01, 0.3, 1.0], rows))


@pytest.mark.parametrize("V", [100, 5000, 40000])
@pytest.mark.parametrize("which", ["none", "temperature", "top_k", "top_p", "min_p"])
def test_one_parameter_alone(srm, which, V):
    rng = np.random.default_rng(V + len(which))
    rows = 40
    kw = {"temperature": rng.uniform(0.2, 3, rows), "top_k": rng.integers(1, V, rows), "top_p": rng.uniform(0.01, 1, rows),
          "min_p": rng.uniform(0, 1, rows) ** 4}
    check(srm, _logits(rng, rows, V), rng.random(rows), **({which: kw[which]} if which != "none" else {}))


def test_flat_rows_and_wide_cuts(srm):
    """Distributions without a peak: thousands of tokens on both sides of the cut, a few of them in every step of logit value."""
    rng = np.random.default_rng(4)
    for V in (3000, 32000, 100000):
        logits = _logits(rng, 12, V, scale=0.01)
        check(srm, logits, rng.random(12), top_p=rng.uniform(0.05, 0.95, 12), top_k=rng.integers(1, V, 12))


@pytest.mark.parametrize("V", [7, 512, 2000, 33000, 140000])
def test_equal_logits(srm, V):
    """Ties go by the index: rows of one value, rows of a few values; cuts inside the ties."""
    rng = np.random.default_rng(V)
    rows = 16
    logits = torch.zeros(rows, V, device="cuda")
    logits[8:] = torch.from_numpy(rng.integers(0, 3, (8, V)).astype(np.float32)).cuda()
    logits[3] = -0.0
    logits[3, ::2] = 0.0
    k = rng.integers(1, V + 1, rows)
    # (strict off: with n equal weights a target of j / n lies on a border exactly, where sums of whole numbers are exact on both sides)
    check(srm, logits, (rng.integers(0, 64, rows) / 64), top_k=k, strict=False)
    check(srm, logits, (rng.integers(0, 64, rows) / 64), top_p=rng.integers(1, 64, rows) / 64 + 1e-4, strict=False)
    check(srm, logits.bfloat16(), rng.random(rows), top_k=k, top_p=rng.uniform(0.1, 1, rows), strict=False)


def test_greedy_takes_the_lowest_index(srm):
    rng = np.random.default_rng(9)
    logits = torch.from_numpy(rng.integers(-3, 3, (30, 9001)).astype(np.float32)).cuda()
    t = np.array([0.0, -1.0, NAN] * 10)
    got = check(srm, logits, rng.random(30), temperature=t, top_k=rng.integers(0, 50, 30), top_p=rng.random(30))
    np.testing.assert_array_equal(got, logits.cpu().numpy().argmax(axis=1))


@pytest.mark.parametrize("V", [5, 700, 32000, 70000])
def test_masked_infinite_and_missing_logits(srm, V):
    rng = np.random.default_rng(V)
    x = rng.standard_normal((14, V)).astype(np.float32)
    x[0] = -INF                                               # nothing left
    x[1] = NAN
    x[2] = -INF
    x[2, V // 2] = -1e30                                      # one token left
    x[3, : V - 1] = -INF                                      # the last one
    x[4] = np.finfo(np.float32).min                           # a mask of the type's lowest value: all alike
    x[5, ::2] = np.finfo(np.float32).min
    x[6, 1] = INF
    x[7, [0, V - 1]] = INF                                    # two share the draw
    x[8, ::3] = NAN
    x[9] = np.where(rng.random(V) < 0.9, -INF, x[9])
    x[10, 0] = 3e38
    x[11] = -3e38
    x[12] *= 1e-30
    x[13, 0] = NAN
    x[13, 1:] = -INF
    logits = torch.from_numpy(x).cuda()
    for kw in ({}, dict(top_k=[3] * 14), dict(top_p=[0.7] * 14), dict(min_p=[0.2] * 14), dict(temperature=[0.0] * 14),
               dict(top_k=[9] * 14, top_p=[0.9] * 14, min_p=[0.001] * 14, temperature=[1.5] * 14)):
        check(srm, logits, [0.37] * 14, strict=False, **kw)
    check(srm, logits.bfloat16(), [0.61] * 14, top_p=[0.8] * 14, strict=False)


def test_values_outside_the_parameters_ranges(srm):
    """What the documentation says of each: off, the nearest allowed value, or greedy."""
    rng = np.random.default_rng(1)
    row = rng.standard_normal(3001).astype(np.float32) * 2
    logits = torch.from_numpy(np.tile(row, (12, 1))).cuda()
    on = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.4)
    cases = [dict(top_k=-5), dict(top_k=2**31 - 1), dict(top_p=2.0), dict(top_p=NAN), dict(top_p=0.0), dict(top_p=-3.0), dict(min_p=NAN),
             dict(min_p=-1.0), dict(min_p=7.0), dict(u=-0.5), dict(u=NAN), dict(u=1.0)]
    meant = [{}, {}, {}, {}, dict(top_k=1), dict(top_k=1), {}, {}, dict(min_p=1.0), dict(u=0.0), dict(u=0.0), dict(u=1.0)]
    col = {k: [{**on, **c}[k] for c in cases] for k in on}
    tok = torch.empty(12, dtype=torch.int32, device="cuda")
    f = torch.float32
    srm.sample_rows(logits, _column(col["u"], f), tok, temperature=_column(col["temperature"], f), top_k=_column(col["top_k"], torch.int32),
                    top_p=_column(col["top_p"], f), min_p=_column(col["min_p"], f))
    want = [fp8_ref.sample(row, **{**on, **m})[0] for m in meant]
    assert want[-1] == 3000 and tok.tolist() == want


@pytest.mark.parametrize("t", [1e-30, 1e-4, 50.0, 1e30, INF])
def test_extreme_temperatures(srm, t):
    rng = np.random.default_rng(2)
    logits = _logits(rng, 8, 6000)
    logits[3, 17] = -INF
    check(srm, logits, rng.random(8), temperature=[t] * 8, top_p=[0.9, 1.0] * 4)


def _odd_rows(rng, V):
    """Rows on which a table of the weights of bf16 logits, with tiny and huge ones apart, could go wrong."""
    x = rng.standard_normal((13, V)) * 2.5
    x[1] *= 4e-4                                              # most magnitudes below 2^-11
    x[2] /= 5
    x[2, ::40] = 0.0
    x[3] = -20.0
    x[3, rng.permutation(V)[:900]] = 0.0                      # limits among the zeros, few enough to be listed
    x[4] = 3.0
    x[5] = rng.choice([2.0, 1.0, -1.0], V)
    x[6] *= 100                                               # magnitudes above 2^9
    x[7] = -np.abs(x[7]) - 1
    x[8, ::2] = -INF
    x[8, 1::50] = NAN
    x[9, V // 3] = INF
    x[10] = rng.uniform(400, 511, V)
    x[11] = rng.uniform(-5e-4, 5e-4, V)
    x[11, ::100] = 4.883e-4                                   # on both sides of 2^-11
    x[12] = np.where(rng.random(V) < 0.5, -510.0, -511.9)
    return x.astype(np.float32)


@pytest.mark.parametrize("V", [6143, 6144, 20479, 20480])
@pytest.mark.parametrize("times", [1, 6])                     # fewer and more rows than compute units
def test_top_p_of_bf16_logits_of_few_or_odd_values(srm, V, times):
    rng = np.random.default_rng(V + times)
    top_p = [0.3, 0.5, 0.9, 0.99, 0.9999, 1.0]
    x = np.concatenate([np.repeat(_odd_rows(rng, V), len(top_p), axis=0) for _ in range(times)])
    rows = len(x)
    check(srm, torch.from_numpy(x).cuda().bfloat16(), rng.random(rows), top_p=top_p * (rows // len(top_p)),
          temperature=np.tile(np.repeat([1.0, 1.0, 0.5, 1.0, 1.0, 0.7, 100.0, 1.0, 1.0, 1.0, 10.0, 1.0, 1.0], len(top_p)), times))


@pytest.mark.parametrize("t", [0.05, 3.0, 11.5, 20.0, 1e4])
def test_temperatures_of_bf16_rows(srm, t):
    """From hot rows whose lowest logit with weight lies below -2^9 to cold ones."""
    rng = np.random.default_rng(31)
    check(srm, _logits(rng, 8, 30000, 0, torch.bfloat16), rng.random(8), temperature=[t] * 8, top_p=[0.9, 1.0] * 4, top_k=[0] * 6 + [700] * 2,
          min_p=[0.0] * 4 + [0.01] * 2 + [0.0] * 2)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,times", [(5, 1), (300, 1), (512, 1), (513, 1), (513, 6), (1000, 6), (1024, 7)])
def test_short_rows_of_few_or_odd_values(srm, V, times, dtype):
    """Equal values at the limits, values of all magnitudes (a search by halves that takes long), masks, infinities, NaN."""
    rng = np.random.default_rng(V)
    x = rng.standard_normal((10, V)) * 2.5
    x[1] = 3.0
    x[2] = rng.choice([2.0, 1.0, -1.0], V)
    x[3] = 10.0 ** rng.uniform(-30, 1, V)
    x[4] = -x[3]
    x[5, ::2] = -INF
    x[5, 1::7] = NAN
    x[6, V // 3:V // 3 + 3] = INF
    x[7] = np.finfo(np.float32).min
    x[7, V // 2] = -3e38
    x[8] = -1e30
    x[8, V // 4:V // 2 + 1] = 4.0
    x[9] = np.where(rng.random(V) < 0.5, 0.0, -0.0)
    x = np.repeat(x.astype(np.float32), 9, axis=0)
    x = torch.from_numpy(np.concatenate([x] * times)).cuda().to(dtype)
    n = x.shape[0]
    check(srm, x, rng.random(n), top_p=[0.3, 0.7, 0.999, 1.0, 1.0, 1.0, 0.5, 0.8, 1.0] * (10 * times), top_k=[0, 0, 0, 3, 200, 1, 4, 250, 0] * (10 * times),
          min_p=[0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.0, 0.01, 0.4] * (10 * times))


def test_an_infinite_temperature_is_the_largest(srm):
    """Of logits that far apart, the probabilities are those of 1e30."""
    x = torch.tensor([[0.0, -2e30], [3e38, -3e38]], device="cuda")
    tok, lp = torch.empty(2, dtype=torch.int32, device="cuda"), torch.empty(2, device="cuda")
    srm.sample_rows(x, _column([0.99, 0.99], torch.float32), tok, temperature=_column([INF, 1e35], torch.float32), logprob=lp)
    want = [float(x[0, 1].double()) / float(np.float32(1e30)), 0.0]
    want[0] -= math.log1p(math.exp(want[0]))
    assert tok.tolist() == [1, 0]
    assert [abs(a - b) <= 2.0 ** -24 * abs(b) + 1e-9 for a, b in zip(lp.double().tolist(), want)] == [True, True]


def test_more_rows_than_a_dimension_of_a_grid_has_threads_for(srm):
    rows, V = (1 << 23) + 3, 5
    logits = torch.randn(rows, V, device="cuda")
    u = torch.rand(rows, device="cuda")
    tok = torch.full((rows + 1,), -7, dtype=torch.int32, device="cuda")
    srm.sample_rows(logits, u, tok[:-1])
    w = torch.exp(logits.double() - logits.double().amax(1, keepdim=True))
    run = w.cumsum(1)
    goal = u.double() * run[:, -1]
    want = (run <= goal[:, None]).sum(1)
    near = ((run - goal[:, None]).abs() < 1e-9).any(1)        # (8 million draws: a few may lie that near)
    assert near.sum() < 10 and tok[-1] == -7
    assert ((tok[:-1] == want) | near).all()


def test_more_work_groups_than_a_row_of_the_grid(srm):
    rows, V = (1 << 21) + 3, 1025
    logits = torch.randn(rows, V, device="cuda", dtype=torch.bfloat16)
    tok = torch.full((rows + 1,), -7, dtype=torch.int32, device="cuda")
    u, cold = torch.rand(rows, device="cuda"), torch.zeros(rows, device="cuda")
    srm.sample_rows(logits, u, tok[:-1], temperature=cold)
    top = logits.amax(1, keepdim=True)
    assert tok[-1] == -7 and int(tok[:-1].amin()) >= 0
    assert torch.equal(logits.gather(1, tok[:-1, None].long()), top)


def test_the_ends_of_the_draw(srm):
    """u = 0 draws the first kept token, the largest u below 1 the last one that has weight."""
    rng = np.random.default_rng(12)
    for V in (10, 8200, 60000):
        logits = _logits(rng, 6, V, scale=1.0)
        check(srm, logits, [0.0] * 6, top_k=[0, 1, 2, 5, 9, 3], strict=False)
        check(srm, logits, [1 - 2.0 ** -24] * 6, top_k=[0, 1, 2, 5, 9, 3])


def test_the_largest_vocabulary_and_many_rows(srm):
    rng = np.random.default_rng(20)
    check(srm, _logits(rng, 2, 1 << 20), rng.random(2), top_p=[0.9, 1.0], top_k=[0, 100000])
    logits = _logits(rng, 3000, 130)
    check(srm, logits, rng.random(3000), top_k=rng.integers(0, 40, 3000), top_p=rng.uniform(0.1, 1, 3000), temperature=rng.uniform(0, 2, 3000))


def test_rows_behind_two_gigabytes(srm):
    V, rows = 131072, 9000                                    # 2.36 GB in bf16, 1.18e9 elements; 4.7 GB in fp32
    rng = np.random.default_rng(21)
    few = _logits(rng, 3, V)
    logits = torch.full((rows, V), -INF, device="cuda")
    at = [0, 4500, rows - 1]
    for r, x in zip(at, few):
        logits[r] = x
    u = torch.full((rows,), 0.3, device="cuda")
    tok = torch.empty(rows, dtype=torch.int32, device="cuda")
    p = torch.full((rows,), 0.9, device="cuda")
    srm.sample_rows(logits, u, tok, top_p=p)
    got = tok.cpu().numpy()
    for r, x in zip(at, few.cpu().numpy()):
        assert got[r] == fp8_ref.sample(x, u=float(np.float32(0.3)), top_p=float(np.float32(0.9)))[0]
    assert (np.delete(got, at) == -1).all()


def test_the_draws_follow_the_distribution(srm):
    """20000 draws of one row with even random numbers: each token's share is its probability, to one draw on either side."""
    row = torch.tensor([0.3, 2.0, -1.0, 1.2, 0.0, -INF, 1.9], device="cuda")
    n = 20000
    u = (torch.arange(n, device="cuda", dtype=torch.float64) / n + 0.5 / n).float()
    tok = torch.empty(n, dtype=torch.int32, device="cuda")
    srm.sample_rows(row.expand(n, 7).contiguous(), u, tok)
    share = torch.bincount(tok.long(), minlength=7).double() / n
    assert (share - torch.softmax(row.double(), 0)).abs().max() <= 2 / n


def test_a_head_in_8_bits_and_its_tokens_captured_and_replayed(srm):
    """The end of a decode step: norm, head, tokens; eager, and as a graph that is replayed with eager calls between."""
    rng = np.random.default_rng(30)
    M, d, V = 19, 256, 4099
    x = torch.randn(M, d, device="cuda")
    gain = torch.ones(d, device="cuda")
    head = srm.fp8_empty(V, d)
    srm.quantize_fp8(torch.randn(V, d, device="cuda") * 0.3, *head)
    q = srm.fp8_empty(M, d)
    logits = torch.empty(M, V, device="cuda")
    tok = torch.empty(M, dtype=torch.int32, device="cuda")
    lp = torch.empty(M, device="cuda")
    u = torch.rand(M, device="cuda")
    cols = dict(temperature=torch.full((M,), 0.7, device="cuda"), top_k=torch.full((M,), 50, dtype=torch.int32, device="cuda"),
                top_p=torch.full((M,), 0.9, device="cuda"), min_p=torch.full((M,), 0.01, device="cuda"))

    def step():
        srm.rmsnorm_fp8(x, gain, 1e-5, *q)
        srm.linear_fp8(4, *q, *head, None, logits)
        srm.sample_rows(logits, u, tok, logprob=lp, **cols)

    inputs = [(torch.randn(M, d, device="cuda"), torch.rand(M, device="cuda")) for _ in range(3)]
    want = []
    for a, b in inputs:
        x.copy_(a)
        u.copy_(b)
        step()
        want.append((tok.clone(), lp.clone()))
        check(srm, logits, u.cpu().numpy(), *(cols[k].cpu().numpy() for k in ("temperature", "top_k", "top_p", "min_p")))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step()
    for i in (1, 0, 2, 1):
        x.copy_(inputs[i][0])
        u.copy_(inputs[i][1])
        srm.sample_rows(logits[:3], u[:3], tok[:3])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tok, want[i][0]) and torch.equal(lp, want[i][1])
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    mine = torch.empty_like(tok)
    srm.sample_rows(logits, u, mine, stream=st, **cols)
    st.synchronize()
    assert torch.equal(mine, want[1][0])
