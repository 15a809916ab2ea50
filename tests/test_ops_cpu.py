"""Refusals of the operators that need no model (8-bit rows, their products, sampling by request), before any HIP call."""
import ctypes as C

import numpy as np
import pytest
import torch

import fp8_ref


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    from paper_2605_08696_amd import build as b
    if b.is_stale():
        b.build_lib()
    pkg.lib()
    return pkg


P = 1 << 20                      # an address that no call may reach
NAN = float("nan")


def refused(srm, rc, word=b""):
    assert rc == -1 and word in srm.lib().srm_last_error(), srm.lib().srm_last_error()


def test_sizes_of_the_format(srm):
    assert [srm.fp8_row_bytes(k) for k in (-1, 0, 1, 128, 129, 4096)] == [0, 0, 128, 128, 256, 4096]
    assert [srm.fp8_scale_bytes(r, k) for r, k in ((0, 5), (3, 0), (1, 1), (3, 512), (3, 513), (1 << 31, 4096))] == \
        [0, 0, 4, 12, 24, (1 << 31) * 32]
    q, s = srm.fp8_empty(3, 513, device="cpu")
    assert q.shape == (3, 640) and s.shape == (2, 3, 4)
    assert q.numel() == 3 * srm.fp8_row_bytes(513) and s.numel() == srm.fp8_scale_bytes(3, 513)


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (0, -1, b"dtype"), (1, None, b"null"), (2, 99, b"stride"), (3, 0, b"sizes"), (3, 1 << 31, b"sizes"),
    (4, 0, b"sizes"), (4, -5, b"sizes"), (4, (1 << 22) + 1, b"sizes"), (5, None, b"null"), (5, P + 8, b"multiples"), (6, None, b"null"),
    (6, P + 2, b"multiples")])
def test_quantize_refuses(srm, at, value, word):
    args = [0, P, 100, 4, 100, P, P, None]
    args[at] = value
    refused(srm, srm.lib().srm_quantize_fp8(*args), word)


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (1, None, b"null"), (2, 99, b"stride"), (3, 7, b"dtype"), (5, 99, b"stride"), (6, None, b"null"), (7, -1.0, b"eps"),
    (7, NAN, b"eps"), (8, 0, b"sizes"), (8, 1 << 31, b"sizes"), (9, 0, b"sizes"), (9, 32769, b"sizes"), (10, None, b"null"),
    (10, P + 1, b"multiples"), (11, None, b"null"), (11, P + 3, b"multiples")])
def test_rmsnorm_refuses(srm, at, value, word):
    args = [0, P, 100, 1, P, 100, P, 1e-5, 4, 100, P, P, None]
    args[at] = value
    refused(srm, srm.lib().srm_rmsnorm_fp8(*args), word)


@pytest.mark.parametrize("at,value,word", [
    (0, 3, b"epilogue"), (0, 5, b"epilogue"), (0, -1, b"epilogue"), (0, 100, b"epilogue"), (1, None, b"null"), (1, P + 8, b"multiples"),
    (2, None, b"null"), (3, None, b"null"), (3, P + 4, b"multiples"), (4, None, b"null"), (4, P + 2, b"multiples"), (5, P + 2, b"element"),
    (6, 0, b"sizes"), (6, 1 << 31, b"sizes"), (7, 0, b"sizes"), (7, -3, b"sizes"), (8, 0, b"sizes"), (8, (1 << 22) + 1, b"sizes"),
    (9, None, b"null"), (9, P + 1, b"element")])
def test_linear_refuses(srm, at, value, word):
    args = [0, P, P, P, P, P, 4, 5, 100, P, None]
    args[at] = value
    refused(srm, srm.lib().srm_linear_fp8(*args), word)
    if at == 9 and value is not None:
        args[0], args[9] = 4, P + 2
        refused(srm, srm.lib().srm_linear_fp8(*args), word)


@pytest.mark.parametrize("at,value,word", [
    (0, 2, b"dtype"), (1, None, b"null"), (2, 99, b"stride"), (3, 0, b"sizes"), (3, 1 << 31, b"sizes"), (4, 0, b"sizes"),
    (4, (1 << 20) + 1, b"sizes"), (9, None, b"null"), (10, None, b"null")])
def test_sample_rows_refuses(srm, at, value, word):
    args = [0, P, 100, 4, 100, None, None, None, None, P, P, None, None]
    args[at] = value
    if at == 4 and value > 100:
        args[2] = value
    refused(srm, srm.lib().srm_sample_rows(*args), word)


@pytest.mark.parametrize("call,args,at", [
    ("srm_quantize_fp8", (0, P, 100, 4, 100, P, P, None), {1: 2}), ("srm_quantize_fp8", (1, P, 100, 4, 100, P, P, None), {1: 1}),
    ("srm_rmsnorm_fp8", (0, P, 100, 1, P, 100, P, 1e-5, 4, 100, P, P, None), {1: 2, 4: 1, 6: 2}),
    ("srm_rmsnorm_fp8", (1, P, 100, 0, P, 100, P, 1e-5, 4, 100, P, P, None), {1: 1, 4: 2, 6: 1}),
    ("srm_sample_rows", (0, P, 100, 4, 100, P, P, P, P, P, P, P, None), {1: 2, 5: 1, 6: 2, 7: 3, 8: 2, 9: 2, 10: 1, 11: 2}),
    ("srm_sample_rows", (1, P, 100, 4, 100, None, None, None, None, P, P, None, None), {1: 1})])
def test_operands_lie_at_whole_elements(srm, call, args, at):
    for i, off in at.items():
        bad = list(args)
        bad[i] = P + off
        refused(srm, getattr(srm.lib(), call)(*bad), b"whole element")


def test_sizes_whose_grids_or_indexes_do_not_fit_are_refused(srm):
    lib, big = srm.lib(), 1 << 30
    refused(srm, lib.srm_quantize_fp8(0, P, 2000, big - 1, 2000, P, P, None), b"sizes")        # 2^32 groups
    refused(srm, lib.srm_quantize_fp8(0, P, 8, big, 8, P, P, None), b"sizes")
    refused(srm, lib.srm_rmsnorm_fp8(0, P, 8, 0, None, 0, P, 0.0, big, 8, P, P, None), b"sizes")
    refused(srm, lib.srm_linear_fp8(0, P, P, P, P, None, big, 1, 1, P, None), b"sizes")
    refused(srm, lib.srm_linear_fp8(0, P, P, P, P, None, 1, big, 1, P, None), b"sizes")
    refused(srm, lib.srm_sample_rows(0, P, 8, big, 8, None, None, None, None, P, P, None, None), b"sizes")


def test_binding_refuses_before_the_library(srm):
    x, add, gain = torch.zeros(3, 200), torch.zeros(3, 200), torch.zeros(200)
    q, s = srm.fp8_empty(3, 200, device="cpu")
    with pytest.raises(ValueError, match="CUDA"):
        srm.quantize_fp8(x, q, s)
    with pytest.raises(ValueError, match="dtype"):
        srm.quantize_fp8(x.double(), q, s)
    with pytest.raises(ValueError, match="matrix"):
        srm.quantize_fp8(x[0], q, s)
    with pytest.raises(ValueError, match="contiguous"):
        srm.quantize_fp8(torch.zeros(200, 3).t(), q, s)
    with pytest.raises(ValueError, match="overlap"):
        srm.quantize_fp8(x[:1].expand(3, 200), q, s)
    with pytest.raises(ValueError, match="shape"):
        srm.quantize_fp8(x, *srm.fp8_empty(3, 300, device="cpu"))
    with pytest.raises(ValueError, match="scales"):
        srm.quantize_fp8(x, q, srm.fp8_empty(3, 600, device="cpu")[1])
    with pytest.raises(ValueError, match="dtypes"):
        srm.quantize_fp8(x, q.view(torch.uint8), s)
    with pytest.raises(ValueError, match="gain"):
        srm.rmsnorm_fp8(x, gain[:-1], 1e-5, q, s)
    with pytest.raises(ValueError, match="add"):
        srm.rmsnorm_fp8(x, gain, 1e-5, q, s, add=add[:2])
    w, ws = srm.fp8_empty(5, 200, device="cpu")
    with pytest.raises(ValueError, match="disagree"):
        srm.linear_fp8(0, q, s, *srm.fp8_empty(5, 300, device="cpu"), None, torch.zeros(3, 5))
    with pytest.raises(ValueError, match="out"):
        srm.linear_fp8(0, q, s, w, ws, None, torch.zeros(3, 5))
    with pytest.raises(ValueError, match="out"):
        srm.linear_fp8(4, q, s, w, ws, None, torch.zeros(3, 6))
    with pytest.raises(ValueError, match="bias"):
        srm.linear_fp8(4, q, s, w, ws, torch.zeros(4), torch.zeros(3, 5))
    tok, u = torch.zeros(3, dtype=torch.int32), torch.zeros(3)
    with pytest.raises(ValueError, match="uniform"):
        srm.sample_rows(x, u[:2], tok)
    with pytest.raises(ValueError, match="top_k"):
        srm.sample_rows(x, u, tok, top_k=u)
    with pytest.raises(ValueError, match="tok_out"):
        srm.sample_rows(x, u, tok.long())
    with pytest.raises(ValueError, match="CUDA"):
        srm.sample_rows(x, u, tok)


def test_the_reference_of_the_format_agrees_with_torch_on_every_code():
    """The tests' own rounding against torch's conversion, at every border between two codes and beside it."""
    codes = torch.arange(0, 0x7F, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    mid = (codes[1:] + codes[:-1]) / 2
    for v in (codes, mid, np.nextafter(mid, 0), np.nextafter(mid, 448)):
        for sign in (1.0, -1.0):
            row = np.full((v.size, 128), 448.0)              # a scale of 1
            row[:, 5] = sign * v
            q, exp = fp8_ref.quantize(row)
            assert (exp == 0).all()
            want = torch.from_numpy(sign * v).float().to(torch.float8_e4m3fn).double().numpy() if v is codes or v is mid else None
            if want is not None:
                np.testing.assert_array_equal(q[:, 5], want)
            else:
                assert (np.abs(q[:, 5] - sign * v) <= np.diff(codes) / 2).all()


def test_the_reference_of_the_rule_on_rows_by_hand():
    L = [0.0, 1.0, 1.0, -np.inf, NAN]
    w = np.exp([-1.0, 0.0, 0.0])
    assert fp8_ref.sample(L, 0.0)[:2] == (1, 0.0)
    assert fp8_ref.sample(L, u=0.0)[0] == 0 and fp8_ref.sample(L, u=w[0] / w.sum() + 1e-9)[0] == 1
    assert fp8_ref.sample(L, u=0.999)[0] == 2 and fp8_ref.sample(L, top_k=1, u=0.999)[0] == 1
    assert fp8_ref.sample(L, top_p=0.4, u=0.999)[0] == 1 and fp8_ref.sample(L, top_p=0.6, u=0.999)[0] == 2
    assert fp8_ref.sample(L, min_p=0.5, u=0.0)[0] == 1 and fp8_ref.sample([-np.inf, NAN])[0] == -1
    assert abs(fp8_ref.sample(L, u=0.0)[1] - np.log(w[0] / w.sum())) < 1e-15
