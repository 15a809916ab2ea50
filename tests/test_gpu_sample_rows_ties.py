"""Sampling by request where limits and draws fall on borders exactly: rows of equal weights, whose rule needs whole numbers only.

Of n equal logits the first k = min(n, top_k) are left by top-k and the first ceil(top_p k) of those, one at least, by top-p; the token is
number floor(u kept) of them.  top_p and u are the fp32 values' exact fractions."""
import math
from fractions import Fraction

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def rule(allowed, u, top_k=0, top_p=1.0):
    """allowed: the indices of the equal logits, in order."""
    kept = min(len(allowed), top_k) if top_k > 0 else len(allowed)
    if top_p < 1:
        kept = max(1, math.ceil(Fraction(float(top_p)) * kept))
    return int(allowed[min(int(Fraction(float(u)) * kept), kept - 1)]), -math.log(kept)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,rows", [(1, 9), (7, 30), (512, 40), (513, 600), (1000, 40), (2000, 300), (6144, 40), (33000, 24), (140000, 12), (1 << 20, 3)])
def test_equal_weights(srm, V, rows, dtype):
    rng = np.random.default_rng(V + rows)
    x = np.full((rows, V), -np.inf, dtype=np.float32)
    allowed = []
    for r in range(rows):
        some = np.arange(V) if r % 3 else np.sort(rng.choice(V, max(1, V // 3), replace=False))
        x[r, some] = (0.0, 3.0, -7.5, 300.0)[r % 4]
        allowed.append(some)
    n = np.array([len(a) for a in allowed])
    # fractions that lie on borders: sixty-fourths, and the fp32 values around j / n
    j = rng.integers(0, n)
    u = np.choose(rng.integers(0, 4, rows), [rng.integers(0, 64, rows) / 64, j / n, np.nextafter((j / n).astype(np.float32), np.float32(1)), rng.random(rows)])
    p = np.choose(rng.integers(0, 4, rows), [rng.integers(1, 65, rows) / 64, (j + 1) / n, np.nextafter(((j + 1) / n).astype(np.float32), np.float32(0)),
                                             rng.random(rows)])
    u, p = np.minimum(u.astype(np.float32), np.float32(1 - 2.0 ** -24)), p.astype(np.float32)
    k = np.where(rng.random(rows) < 0.4, 0, rng.integers(1, V + 2, rows)).astype(np.int32)
    on = torch.full((rows,), 0.7, device="cuda")
    dev = [torch.from_numpy(a).cuda() for a in (x, u, k, p)]
    dev[0] = dev[0].to(dtype)
    tok, lp = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    for with_k in (False, True):
        for with_p in (False, True):
            print(f"sample_rows of equal weights {dtype} {rows} x {V}, top_k {with_k}, top_p {with_p}", flush=True)
            srm.sample_rows(dev[0], dev[1], tok, temperature=on, top_k=dev[2] if with_k else None, top_p=dev[3] if with_p else None, logprob=lp)
            got, gl = tok.cpu().numpy(), lp.double().cpu().numpy()
            for r in range(rows):
                want, logp = rule(allowed[r], u[r], int(k[r]) if with_k else 0, p[r] if with_p else 1.0)
                assert got[r] == want, (r, n[r], u[r], k[r], p[r], got[r], want)
                assert abs(gl[r] - logp) <= 2.0 ** -24 * abs(logp) * 1.01 + 1e-9, (r, gl[r], logp)
