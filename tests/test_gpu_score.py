"""Scores of given tokens through the public binding, against the same in 64 bits (recur_ref.score).  Tokens have to be equal.  Z is a sum
of V weights, each off by its argument's roundings (|d| up to some 90 at 2^-23: 3e-6 of a weight e^-d, which is below 2^-22 of the sum) and
summed by a thread and over threads: (V / 256 + 40) 2^-24 of it at most; the logarithm 2^-22 of its value, and log p one rounding of
|d| + log Z (3 2^-24 of it).  The entropy has a second such sum, relative to its own size."""
import math

import numpy as np
import pytest
import torch

import recur_ref

pytestmark = pytest.mark.gpu
INF, NAN = math.inf, math.nan


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def check(srm, logits, token, top, temperature=None):
    rows, V = logits.shape
    token = torch.tensor(np.asarray(token), dtype=torch.int32, device="cuda")
    temp = None if temperature is None else torch.tensor(np.asarray(temperature), dtype=torch.float32, device="cuda")
    lp, en = (torch.full((rows + 2,), 7.0, device="cuda") for _ in range(2))
    tt = torch.full((rows + 2, top), -7, dtype=torch.int32, device="cuda") if top else None
    tl = torch.full((rows + 2, top), 7.0, device="cuda") if top else None
    print(f"token_logprobs {logits.dtype} {rows} x {V}, stride {logits.stride(0)}, top {top}", flush=True)
    srm.token_logprobs(logits, token, lp[1:-1], temperature=temp, entropy=en[1:-1], top_token=tt[1:-1] if top else None, top_logprob=tl[1:-1] if top else None)
    torch.cuda.synchronize()
    for t, v in ((lp, 7), (en, 7), (tt, -7), (tl, 7)):
        if t is not None:
            assert (t[0] == v).all() and (t[-1] == v).all()
    host = logits.double().cpu()
    rel = (V / 256 + 48) * 2.0 ** -24
    for r in range(rows):
        t = 1.0 if temp is None else temp[r].item()
        want, entropy, tokens, logs = recur_ref.score(host[r], int(token[r]), top, t)

        def near(got, ref, what):
            if abs(ref) >= 2.0 ** 128 - 2.0 ** 103:            # rounds to infinity in fp32
                assert got == math.copysign(INF, ref), (what, r, got, ref)
            else:
                assert abs(got - ref) <= rel + 4 * 2.0 ** -24 * (abs(ref) + math.log(V) + 1), (what, r, got, ref)

        near(lp[1 + r].item(), want, "logprob")
        got = en[1 + r].item()
        assert abs(got - entropy) <= rel * (1 + 2 * entropy) + 8 * 2.0 ** -24 * (entropy + math.log(V) + 1), ("entropy", r, got, entropy)
        if top:
            assert tt[1 + r].tolist() == tokens, r
            for k in range(top):
                near(tl[1 + r, k].item(), logs[k], "top")


def _logits(rng, rows, V, pad=0, dtype=torch.float32, offset=0, scale=3.0):
    flat = torch.zeros(offset + rows * (V + pad), dtype=dtype, device="cuda")
    t = flat[offset:].view(rows, V + pad)
    t.copy_(torch.from_numpy((rng.standard_normal((rows, V + pad)) * scale).astype(np.float32)))
    return t[:, :V]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,pad,offset", [(1, 0, 0), (2, 1, 0), (7, 0, 1), (8, 3, 0), (9, 0, 0), (31, 0, 1), (64, 3, 0), (513, 0, 0), (1000, 5, 3), (2048, 0, 0), (8192, 0, 0),
                                          (8193, 0, 1), (32000, 0, 0), (32769, 8, 0), (50021, 1, 2), (150001, 0, 1)])
def test_rows_of_every_length(srm, V, pad, offset, dtype):
    rng = np.random.default_rng(V)
    for rows, top in ((1, 20), (5, 32), (7, 1), (4, 0)):
        logits = _logits(rng, rows, V, pad, dtype, offset)
        check(srm, logits, rng.integers(-1, V + 1, rows), top, rng.choice([0.3, 0.7, 1.0, 2.0], rows) if top == 32 else None)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 5, 40, 3000, 40000])
def test_masks_infinities_nan_and_equal_logits(srm, V, dtype):
    rng = np.random.default_rng(V + 1)
    x = (rng.standard_normal((16, V)) * 3).astype(np.float32)
    x[0] = -INF                                                # nothing left
    x[1] = NAN
    x[2, rng.random(V) < 0.9] = -INF
    x[3, rng.random(V) < 0.5] = NAN
    x[4, V // 2] = INF
    x[5, ::2] = INF                                            # in bulk
    x[6] = 1.25                                                # all equal
    x[7] = rng.integers(0, 2, V)
    x[8] = np.where(np.arange(V) % 2, -0.0, 0.0)
    x[9] = np.arange(V)                                        # the largest ones side by side
    x[10] = -np.arange(V)
    x[11] = np.finfo(np.float32).min                           # masks of the lowest value
    x[11, V // 3] = 0.0
    x[12] = -INF
    x[12, V - 1] = -3.0e38
    x[13] *= 1e30
    x[14, V // 2:] = 2.5
    logits = torch.from_numpy(x).to(dtype).cuda()
    token = [0, V - 1, V // 2, V // 3, V // 2, min(V - 1, 1), V - 1, V - 1, 0, V - 1, 0, V // 3, V - 1, V - 1, V, -100]
    for top in (0, 3, 32):
        check(srm, logits, token, top)
    check(srm, logits, token, 20, [0.0, -1.0, NAN, 1e-40, 0.5, 0.5, 2.0, 1e-3, 1.0, 1e-3, 1e38, 0.7, 0.7, 1e33, 0.1, INF])


def test_a_threads_own_logits_are_the_largest(srm):
    """The largest logits lie where one thread reads, so that all but one of the groups' largest are low."""
    V = 40000
    x = np.zeros((3, V), dtype=np.float32)
    x[0, 8:16] = np.arange(8)
    for k in range(V // 8192 + 1):
        x[1, k * 8192 + 40:k * 8192 + 48] = 5 + np.arange(8) + k
    x[2, 32768 - 24:32768] = 9.0
    check(srm, torch.from_numpy(x).cuda(), [8, 40, 5], 32)


def test_outputs_one_by_one(srm):
    rng = np.random.default_rng(2)
    logits, token = _logits(rng, 5, 900), torch.arange(5, dtype=torch.int32, device="cuda")
    lp, en = torch.empty(5, device="cuda"), torch.empty(5, device="cuda")
    tt, tl = torch.empty(5, 4, dtype=torch.int32, device="cuda"), torch.empty(5, 4, device="cuda")
    srm.token_logprobs(logits, token, lp, entropy=en, top_token=tt, top_logprob=tl)
    lp2, en2, tt2, tl2 = (torch.empty_like(t) for t in (lp, en, tt, tl))
    srm.token_logprobs(logits, token, lp2)
    srm.token_logprobs(logits, None, None, entropy=en2)
    srm.token_logprobs(logits, None, None, top_token=tt2, top_logprob=tl2)
    torch.cuda.synchronize()
    assert torch.equal(lp, lp2) and torch.equal(en, en2) and torch.equal(tt, tt2) and torch.equal(tl, tl2)
