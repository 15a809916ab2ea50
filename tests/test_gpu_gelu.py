"""The GELU of the products' epilogues over all of fp32's range: far tails, infinities, NaN.

x Phi(x) is 0 for x = -infinity and below about -40 to any type's last bit, x itself above 7 to bf16's.  Its fitted form for bf16 outputs is
within 6.5e-7 of it, and the output rounds by 2^-8 of its value."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")
ENDS = [0.0, -0.0, 1e-30, -1e-30, 0.5, -0.5, 3.0, -3.0, 5.5, -5.5, 6.08, -6.08, 6.1, -6.1, 7.0, -7.0, 12.0, -12.0, 100.0, -100.0, 1e3, -1e3, 1e4, -1e4,
        1e6, -1e6, 1e15, -1e15, 1e30, -1e30, 3.3e38, -3.3e38, INF, -INF, NAN, 2.0]


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def check_gelu(out, x):
    """out: bf16; x: what went in, fp64."""
    want = torch.where(x == -INF, 0.0, x * torch.special.ndtr(x))
    got = out.double()
    wrong = (got.isnan() != want.isnan()).nonzero()
    assert len(wrong) == 0, [(i, float(x[tuple(i)]), float(got[tuple(i)])) for i in wrong[:8].tolist()]
    # (3.3e38 rounds to 3.29e38 in bf16: nothing finite becomes infinite)
    assert torch.equal(got.isinf(), want.isinf()) and (got[got.isinf()] == want[want.isinf()]).all()
    some = want.isfinite()
    off = (got - want).abs() - (6.5e-7 + 2.0 ** -8 * want.abs())
    assert (off[some] <= 0).all(), (float(off[some].max()), float(x[some][off[some].argmax()]))


def _ends(N):
    return torch.tensor(np.resize(np.array(ENDS, dtype=np.float32), N), device="cuda")


# K cut over the wavefronts, tiles, the persistent 256x256 kernel
@pytest.mark.parametrize("M,N,K", [(5, 72, 128), (33, 520, 256), (1100, 1028, 256), (2048, 2048, 128), (4096, 4096, 256)])
def test_linear_fp8(srm, M, N, K):
    """Sums that are the bias alone, and in rows 1 to 4 infinite or NaN ones.  Rows 1 and 2 hold the products +-448^2 2^200 = 3e65, beyond
    fp32 but finite: with a bias of the opposite infinity the sum is that infinity where one instruction adds both, and NaN where the
    products are rounded to fp32 first.  Either may come, so those elements are looked at apart."""
    a, sa = srm.fp8_empty(M, K)
    w, sw = srm.fp8_empty(N, K)
    a.view(torch.uint8).zero_()
    w.view(torch.uint8).fill_(0x7E)                           # 448
    for s in (sa, sw):
        s.view(torch.uint8).fill_(127)
    sw.view(torch.uint8).fill_(227)                           # 2^100
    sa.view(torch.uint8)[0, 1:3] = 227
    a.view(torch.uint8)[1, 3] = 0x7E
    a.view(torch.uint8)[2, 3] = 0xFE
    a.view(torch.uint8)[3, 3] = 0x7F                          # NaN
    a.view(torch.uint8)[4, 70] = 0x38                         # 1
    bias = _ends(N)
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    print(f"linear_fp8 with GELU {M} x {N} x {K}", flush=True)
    srm.linear_fp8(1, a, sa, w, sw, bias, out)
    torch.cuda.synchronize()
    x = bias.double().expand(M, N).clone()
    x[1] += INF
    x[2] -= INF
    x[3] = NAN
    x[4] = (x[4] + 448 * 2.0 ** 100).float().double()
    for r, opposite in ((1, -INF), (2, INF)):
        both = bias == opposite
        got = out[r][both].double()
        assert (got.isnan() | (got == max(opposite, 0.0)) | (got.abs() <= (6.5e-7 if opposite < 0 else 0.0))).all()
        out[r][both], x[r][both] = 0.0, 0.0
    check_gelu(out, x)


@pytest.mark.parametrize("M,N,K", [(1, 72, 64), (5, 512, 128), (37, 4096, 1024), (300, 1024, 256), (1100, 1028, 256), (4096, 4096, 128)])
def test_linear(srm, M, N, K):
    """The same of the bf16 products, by a bias."""
    A = torch.zeros(M, K, dtype=torch.bfloat16, device="cuda")
    W = torch.ones(N, K, dtype=torch.bfloat16, device="cuda")
    bias = _ends(N)
    out = torch.empty(M, N, dtype=torch.bfloat16, device="cuda")
    print(f"linear with GELU {M} x {N} x {K}", flush=True)
    srm.linear(srm.SRM_BF16, 1, A, W, bias, out=out)
    torch.cuda.synchronize()
    check_gelu(out, bias.double().expand(M, N))
