"""Refusals of the short convolution, the selective scan and step and the scores of tokens, before any HIP call; and their references."""
import math

import numpy as np
import pytest
import torch

import recur_ref


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    from paper_2605_08696_amd import build as b
    if b.is_stale():
        b.build_lib()
    pkg.lib()
    return pkg


P = 1 << 20                      # an address that no call may reach


def refused(srm, rc, word=b""):
    assert rc == -1 and word in srm.lib().srm_last_error(), srm.lib().srm_last_error()


def host(*values):
    a = np.array(values, dtype=np.int32)
    host.kept = a
    return a.ctypes.data


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (0, -1, b"dtype"), (1, None, b"null"), (1, P + 1, b"element"), (2, 99, b"stride"), (3, None, b"null"), (3, P + 2, b"element"),
    (4, P + 1, b"element"), (5, 2, b"activation"), (6, 0, b"sizes"), (6, (1 << 24) + 1, b"sizes"), (7, 0, b"sizes"), (7, 9, b"sizes"), (8, None, b"null"),
    (9, None, b"null"), (9, P + 2, b"element"), (10, 0, b"sizes"), (10, -1, b"sizes"), (11, P + 1, b"element"), (12, P + 3, b"element"),
    (13, -1, b"sizes"), (13, 0, b"sizes"), (14, P + 1, b"element"), (15, None, b"null"), (15, P + 1, b"element"), (16, 99, b"stride")])
def test_conv_refuses(srm, at, value, word):
    args = [1, P, 100, P, P, 1, 100, 4, host(0, 5), P, 1, P, P, 3, P, P, 100, None]
    args[at] = value
    refused(srm, srm.lib().srm_causal_conv(*args), word)


@pytest.mark.parametrize("offsets,word", [((-1, 5), b"negative"), ((3, 2), b"fall"), ((0, 5, 4, 9), b"fall"), ((0, 1 << 30), b"sizes"),
                                          ((0, 2 ** 31 - 1), b"sizes")])
def test_offsets_are_refused(srm, offsets, word):
    n = len(offsets) - 1
    refused(srm, srm.lib().srm_causal_conv(1, P, 8, P, P, 1, 8, 4, host(*offsets), P, n, None, None, 0, None, P, 8, None), word)
    refused(srm, srm.lib().srm_selective_scan(1, P, 24, 0, P, 2, P, P, P, 1, None, 0, 2, 4, 1, 8, host(*offsets), P, n, None, None, 0, None, P, 8, None, 0,
                                              None), word)
    assert srm.lib().srm_selective_scan_workspace_bytes(1, host(*offsets), n, 2, 4, 8) == 0


SCAN = [1, P, 24, 0, P, 2, P, P, P, 1, P, 8, 2, 4, 1, 8, "offsets", P, 1, P, P, 3, P, P, 8, P, 0, None]


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (1, None, b"null"), (1, P + 1, b"element"), (2, 23, b"stride"), (3, 5, b"dtype"), (4, None, b"null"), (4, P + 2, b"element"), (5, 1, b"stride"),
    (6, None, b"null"), (6, P + 2, b"element"), (7, P + 2, b"element"), (8, P + 1, b"element"), (10, P + 1, b"element"), (11, 7, b"stride"), (12, 0, b"sizes"),
    (12, 65537, b"sizes"), (13, 0, b"sizes"), (13, 4097, b"sizes"), (14, 0, b"sizes"), (14, 3, b"sizes"), (15, 0, b"sizes"), (15, 257, b"sizes"), (16, None, b"null"),
    (17, None, b"null"), (17, P + 1, b"element"), (18, 0, b"sizes"), (19, P + 2, b"element"), (20, P + 2, b"element"), (21, 0, b"sizes"), (21, -4, b"sizes"),
    (22, P + 2, b"element"), (23, None, b"null"), (23, P + 1, b"element"), (24, 7, b"stride"), (25, P + 2, b"element")])
def test_scan_refuses(srm, at, value, word):
    args = list(SCAN)
    args[16] = host(0, 5)
    args[at] = value
    refused(srm, srm.lib().srm_selective_scan(*args), word)


STEP = [1, P, 24, P, P, 1, 4, P, 0, P, 2, P, P, P, 1, P, 8, 2, 4, 1, 8, 5, P, P, 3, P, P, 8, None]


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (1, None, b"null"), (1, P + 1, b"element"), (2, 23, b"stride"), (3, P + 2, b"element"), (4, P + 2, b"element"), (5, -1, b"activation"),
    (6, 0, b"sizes"), (6, 9, b"sizes"), (7, None, b"null"), (7, P + 1, b"element"), (8, 3, b"dtype"), (9, None, b"null"), (10, 1, b"stride"), (11, None, b"null"),
    (16, 7, b"stride"), (17, 0, b"sizes"), (18, 0, b"sizes"), (19, 3, b"sizes"), (20, 257, b"sizes"), (21, 0, b"sizes"), (21, 1 << 31, b"sizes"), (22, None, b"null"),
    (22, P + 2, b"element"), (23, P + 1, b"element"), (24, 0, b"sizes"), (25, None, b"null"), (25, P + 2, b"element"), (26, None, b"null"), (27, 7, b"stride")])
def test_step_refuses(srm, at, value, word):
    args = list(STEP)
    args[at] = value
    refused(srm, srm.lib().srm_selective_step(*args), word)


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (1, None, b"null"), (1, P + 2, b"element"), (2, 99, b"stride"), (3, 0, b"sizes"), (3, 1 << 31, b"sizes"), (4, 0, b"sizes"),
    (5, P + 1, b"element"), (6, None, b"null"), (6, P + 2, b"element"), (7, None, b"null"), (7, P + 2, b"element"), (8, P + 2, b"element"), (9, -1, b"sizes"),
    (9, 33, b"sizes"), (10, None, b"null"), (10, P + 1, b"element"), (11, None, b"null"), (11, P + 2, b"element")])
def test_token_logprobs_refuses(srm, at, value, word):
    args = [0, P, 100, 4, 100, P, P, P, P, 5, P, P, None]
    args[at] = value
    refused(srm, srm.lib().srm_token_logprobs(*args), word)
    args = [0, P, 100, 4, 100, None, None, None, None, 0, None, None, None]
    refused(srm, srm.lib().srm_token_logprobs(*args), b"nothing")


def test_grids_that_do_not_fit_are_refused(srm):
    lib = srm.lib()
    refused(srm, lib.srm_causal_conv(1, P, 1 << 24, P, P, 1, 1 << 24, 4, host(0, 1 << 29), P, 1, None, None, 0, None, P, 1 << 24, None), b"sizes")
    refused(srm, lib.srm_selective_step(1, P, 1 << 28, None, None, 0, 0, None, 0, P, 65536, P, P, P, 1, None, 0, 65536, 64, 1, 64, 1 << 20, P, None, 1, P, P,
                                        1 << 28, None), b"sizes")
    refused(srm, lib.srm_selective_scan(1, P, 1 << 30, 0, P, 65536, P, P, P, 1, None, 0, 65536, 1 << 14, 1, 8, host(0, 5), P, 1, None, None, 0, None, P, 1 << 30,
                                        None, 0, None), b"sizes")


def test_no_rows_is_no_work(srm):
    """Only empty sequences: nothing is launched."""
    lib = srm.lib()
    assert lib.srm_causal_conv(1, P, 8, P, P, 1, 8, 4, host(3, 3, 3), P, 2, None, None, 0, None, P, 8, None) == 0
    args = list(SCAN)
    args[16], args[18] = host(0, 0), 1
    assert lib.srm_selective_scan(*args) == 0


def test_the_workspace_is_for_few_long_sequences(srm):
    def need(*lengths, heads=32, dim=64, state=128):
        return srm.selective_scan_workspace_bytes(srm.SRM_BF16, np.concatenate([[0], np.cumsum(lengths)]), heads, dim, state)
    assert need(37) == 0 and need(*[300] * 64) == 0
    one = (2 * 64 * 128 + 1) * 32 * 4
    assert need(16384) > 0 and need(16384) % one == 0
    assert srm.selective_scan_workspace_bytes(7, np.array([0, 16384]), 32, 64, 128) == 0
    assert srm.selective_scan_workspace_bytes(1, np.array([0, 16384]), 32, 64, 257) == 0


def test_binding_refuses_before_the_library(srm):
    bf = torch.bfloat16
    x, w, out = torch.zeros(5, 24, dtype=bf), torch.zeros(24, 4), torch.zeros(5, 24, dtype=bf)
    off, d_off = [0, 5], torch.tensor([0, 5], dtype=torch.int32)

    def bad(match, fn, *args, **kw):
        with pytest.raises(ValueError, match=match):
            fn(*args, **kw)

    conv = srm.causal_conv
    bad("CUDA", conv, x, w, None, off, d_off, out)
    bad("weight", conv, x, w[:-1], None, off, d_off, out)
    bad("weight", conv, x, w.flatten(), None, off, d_off, out)
    bad("bias", conv, x, w, torch.zeros(23), off, d_off, out)
    bad("rows", conv, x, w, None, [0, 6], torch.tensor([0, 6], dtype=torch.int32), out)
    bad("boundaries", conv, x, w, None, [0], d_off[:1], out)
    bad("d_offsets", conv, x, w, None, off, d_off.long(), out)
    bad("d_offsets", conv, x, w, None, [0, 2, 5], d_off, out)
    bad("out", conv, x, w, None, off, d_off, out.float())
    bad("out", conv, x, w, None, off, d_off, out[:4])
    bad("pos", conv, x, w, None, off, d_off, out, pos=d_off)
    bad("slot", conv, x, w, None, off, d_off, out, slot=d_off)
    bad("state", conv, x, w, None, off, d_off, out, state=torch.zeros(2, 24, 4, dtype=bf))
    bad("state", conv, x, w, None, off, d_off, out, state=torch.zeros(2, 4, 24))
    bad("dtype", conv, x.half(), w, None, off, d_off, out.half())

    dt, a, y = torch.zeros(5, 2), torch.zeros(2), torch.zeros(5, 8, dtype=bf)
    scan = srm.selective_scan
    bad("CUDA", scan, x, dt, a, off, d_off, y)
    bad("heads", scan, x, dt, a, off, d_off, y, groups=3)
    bad("heads", scan, x, dt, a, off, d_off, torch.zeros(5, 7, dtype=bf))
    bad("columns", scan, x[:, :23], dt, a, off, d_off, y)
    bad("columns", scan, x[:, :8], dt, a, off, d_off, y)
    bad("dt", scan, x, dt[:, :1], a, off, d_off, y)
    bad("dt_bias", scan, x, dt, a, off, d_off, y, dt_bias=torch.zeros(3))
    bad("skip", scan, x, dt, a, off, d_off, y, skip=torch.zeros(2, dtype=bf))
    bad("z", scan, x, dt, a, off, d_off, y, z=torch.zeros(5, 8))
    bad("state", scan, x, dt, a, off, d_off, y, state=torch.zeros(1, 2, 4, 7))
    bad("workspace", scan, x, dt, a, off, d_off, y, workspace=torch.zeros(5))
    step, pos = srm.selective_step, torch.zeros(5, dtype=torch.int32)
    state, ring = torch.zeros(6, 2, 4, 8), torch.zeros(6, 4, 24, dtype=bf)
    bad("CUDA", step, x, dt, a, pos, state, y, weight=w, conv_state=ring)
    bad("pos", step, x, dt, a, pos[:4], state, y)
    bad("state", step, x, dt, a, pos, state.to(bf), y)
    bad("conv_state", step, x, dt, a, pos, state, y, weight=w, conv_state=ring[:5])
    bad("conv_state", step, x, dt, a, pos, state, y, weight=w, conv_state=ring.float())
    bad("weight", step, x, dt, a, pos, state, y, weight=w.to(bf), conv_state=ring)

    logits, token, lp = torch.zeros(3, 50), torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    score = srm.token_logprobs
    bad("CUDA", score, logits, token, lp)
    bad("token", score, logits, token.long(), lp)
    bad("logprob", score, logits, token, lp[:2])
    bad("entropy", score, logits, token, lp, entropy=lp.double())
    bad("temperature", score, logits, token, lp, temperature=lp[:1])
    bad("top", score, logits, token, lp, top_token=torch.zeros(3, 4, dtype=torch.int32))
    bad("top_logprob", score, logits, token, lp, top_token=torch.zeros(3, 4, dtype=torch.int32), top_logprob=torch.zeros(3, 5))


def test_the_references_by_hand():
    x = torch.tensor([[1.0], [2.0], [3.0]])
    w = torch.tensor([[10.0, 1.0]])
    ring = torch.tensor([[[5.0], [7.0]]])
    out, _, _, after = recur_ref.conv(x, w, None, [0, 3], [3], [0], ring, False)
    assert out[:, 0].tolist() == [51.0, 12.0, 23.0] and after[0, :, 0].tolist() == [2.0, 3.0]     # read: position 2, row 0; left: 4 in row 0, 5 in row 1
    out, _, _, after = recur_ref.conv(x, w, None, [0, 0, 3], [0, 0], [0, -1], ring, False)
    assert out[:, 0].tolist() == [1.0, 12.0, 23.0] and torch.equal(after, ring.double())
    xbc, dt, a = torch.tensor([[2.0, 3.0, 5.0], [1.0, 1.0, 1.0]]), torch.ones(2, 1), torch.tensor([-math.log(2.0)])
    y, _, state, _ = recur_ref.scan(xbc, dt, a, [0, 2], 1, 1, 1, 1, softplus=False, state=torch.tensor([[[[8.0]]]]), pos=[1])
    assert torch.allclose(y[:, 0], torch.tensor([50.0, 6.0], dtype=torch.float64)) and abs(state.item() - 6.0) < 1e-6
    lp, en, tok, logs = recur_ref.score(torch.tensor([0.0, math.log(3.0), -math.inf, math.nan]), 0, 3)
    assert abs(lp + math.log(4)) < 1e-6 and tok == [1, 0, -1] and logs[2] == -math.inf
    assert abs(en - (0.25 * math.log(4) + 0.75 * math.log(4 / 3))) < 1e-6
