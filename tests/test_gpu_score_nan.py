"""Scores of rows that hold NaN of all kinds, signalling ones among them: each counts as -infinity, wherever it lies beside other logits."""
import numpy as np
import pytest
import torch

from test_gpu_score import check, srm  # noqa: F401

pytestmark = pytest.mark.gpu
KINDS = {torch.float32: (torch.int32, [0x7F800001, 0x7FBFFFFF, 0x7FC00000, -0x007FFFFF, -1]),
         torch.bfloat16: (torch.int16, [0x7F81, 0x7FBF, 0x7FC0, -0x007F, -1])}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [8, 43, 3000, 20011, 40000])
def test_a_nan_beside_the_rows_largest_logit(srm, V, dtype):  # noqa: F811
    """One NaN at each of eight neighbouring places, whose others hold the row's largest logits; then all places but one."""
    rng = np.random.default_rng(V)
    whole, kinds = KINDS[dtype]
    rows = [(i, k) for i in range(8) for k in range(len(kinds))]
    at = 0 if V < 16 else (V // 2) // 8 * 8
    logits = torch.from_numpy((rng.standard_normal((2 * len(rows), V)) * 2).astype(np.float32)).to(dtype)
    logits[:, at:at + 8] = torch.from_numpy(20 + 2 * rng.permuted(np.tile(np.arange(8), (2 * len(rows), 1)), axis=1)).to(dtype)
    bits = logits.view(whole)
    for r, (i, k) in enumerate(rows):
        bits[2 * r, at + i] = kinds[k]
        kept = bits[2 * r + 1, at + i].clone()
        bits[2 * r + 1, at:at + 8] = torch.tensor([kinds[(k + j) % len(kinds)] for j in range(8)], dtype=whole)
        bits[2 * r + 1, at + i] = kept
    assert logits.isnan().sum() == len(rows) * 8
    check(srm, logits.cuda(), [at + r % 8 for r in range(2 * len(rows))], 5 if V > 8 else 8)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_nan_everywhere_but_in_a_few_places(srm, dtype):  # noqa: F811
    rng = np.random.default_rng(5)
    whole, kinds = KINDS[dtype]
    V = 35000
    logits = torch.zeros(6, V, dtype=dtype)
    bits = logits.view(whole)
    bits.copy_(torch.from_numpy(rng.choice(np.array(kinds), (6, V))).to(whole))
    for r in range(1, 6):                                      # (row 0: nothing left)
        where = torch.from_numpy(rng.choice(V, 10 ** (r - 1), replace=False))
        logits[r, where] = torch.from_numpy(rng.standard_normal(10 ** (r - 1)).astype(np.float32) * 3).to(dtype) if r < 5 else 1.0
    check(srm, logits.cuda(), [0, 1, 2, 3, 4, 5], 20)
