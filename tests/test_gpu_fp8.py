"""Rows in 8 bits and their products through the public binding, against 64-bit references.

Tolerances count roundings.  fp32 rounds by 2^-24 of a value, bf16 by 2^-8, e4m3 by 2^-4 (half a step of its three mantissa bits)
above 2^-6 and by 2^-10 below, in units of a block's scale."""
import numpy as np
import pytest
import torch

import fp8_ref

pytestmark = pytest.mark.gpu
TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _wide(rng, rows, d, pad, dtype, offset=0, scale=1.0):
    """[rows][d] with `pad` elements between rows, `offset` elements behind an allocation's start; some columns ten times as large."""
    a = rng.standard_normal((rows, d)).astype(np.float32) * scale
    a[:, 3 % d::41] *= 10
    flat = torch.zeros(offset + rows * (d + pad), dtype=dtype, device="cuda")
    t = flat[offset:].view(rows, d + pad)[:, :d]
    t.copy_(torch.from_numpy(a))
    return t


def _empty(srm, rows, K):
    """An fp8 matrix inside larger buffers whose other bytes are checked afterwards."""
    q, s = srm.fp8_empty(rows, K)
    qb = torch.full((q.numel() + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    sb = torch.full((s.numel() + 256,), 0x5A, dtype=torch.uint8, device="cuda")
    q = qb[128:-128].view(q.shape).view(torch.float8_e4m3fn)
    s = sb[128:-128].view(s.shape).view(torch.float8_e8m0fnu)

    def untouched():
        for b in (qb, sb):
            assert (b[:128] == 0x5A).all() and (b[-128:] == 0x5A).all()
    return q, s, untouched


def _host(t):
    return t.detach().double().cpu().numpy()


def _words(s):
    return s.view(torch.uint8).cpu().numpy()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("rows,d,pad,offset", [
    (1, 1, 0, 0), (3, 2, 0, 1), (1, 127, 0, 0), (2, 128, 0, 0), (5, 129, 3, 0), (4, 511, 1, 1), (7, 512, 0, 0), (3, 513, 0, 3), (64, 1000, 8, 0),
    (1, 4096, 0, 0), (37, 4096, 0, 0), (33, 4097, 2, 5), (260, 640, 0, 0), (2, 70000, 0, 0), (4099, 1030, 0, 1), (130, 7, 0, 0), (1000, 64, 5, 1), (77, 100, 0, 0), (70, 129, 1, 1), (41, 255, 0, 0),
    (19, 256, 0, 0), (35, 257, 0, 0)])
def test_quantize_has_the_bits_of_the_format(srm, dtype, rows, d, pad, offset):
    rng = np.random.default_rng(rows * 1000 + d)
    x = _wide(rng, rows, d, pad, TYPES[dtype], offset)
    q, s, untouched = _empty(srm, rows, d)
    print(f"quantize {dtype} {rows} x {d} + {pad}, offset {offset}", flush=True)
    srm.quantize_fp8(x, q, s)
    torch.cuda.synchronize()
    untouched()
    want, exp = fp8_ref.quantize(_host(x))
    np.testing.assert_array_equal(_words(s), fp8_ref.scale_words(exp))
    np.testing.assert_array_equal(_host(q.float()), want)


def test_quantize_at_the_ends_of_the_types(srm):
    """Blocks of zeros, of subnormals, of the largest values; a largest value at and beside a border between two scales; ties of e4m3's
    rounding; infinities and NaN, which become NaN without moving the scale."""
    rng = np.random.default_rng(5)
    tiny = np.float32(1e-45)
    x = np.zeros((12, 512), dtype=np.float32)
    x[1] = tiny * rng.integers(-1000, 1000, 512)
    x[2] = 3.4e38 * rng.uniform(-1, 1, 512)
    x[3] = np.float32(2.0) ** rng.integers(-140, 127, 512)
    x[4, ::128] = 448.0
    x[5, ::128] = np.nextafter(np.float32(448.0), np.float32(1000.0))
    x[6, ::128] = np.nextafter(np.float32(448.0), np.float32(0.0))
    x[4:7, 1::128] = 2.0 ** -9                                # e4m3's smallest, at a scale of 1
    x[4:7, 2::128] = 2.0 ** -10                               # a tie between it and zero
    x[4:7, 3::128] = 3 * 2.0 ** -10
    x[4:7, 4::128] = -17.0                                    # a tie between 16 and 18
    x[4:7, 5::128] = 19.0
    x[7] = rng.standard_normal(512)
    x[7, 7], x[7, 130], x[7, 300] = np.inf, -np.inf, np.nan
    x[8] = np.nan
    x[9] = np.inf
    x[10, 5] = -2.0 ** -126
    x[11] = -0.0
    t = torch.from_numpy(x).cuda()
    q, s, untouched = _empty(srm, 12, 512)
    srm.quantize_fp8(t, q, s)
    torch.cuda.synchronize()
    untouched()
    want, exp = fp8_ref.quantize(x.astype(np.float64))
    np.testing.assert_array_equal(_words(s), fp8_ref.scale_words(exp))
    np.testing.assert_array_equal(_host(q.float()), want)


def check_norm(x, gain, eps, q, s, d):
    """q, s against the norm of x (64 bits): every value within half a step of e4m3 and the roundings of fp32 in front of it."""
    v = _host(x)
    y = v / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps) * _host(gain)
    blocks = q.shape[1] // 128
    exp = fp8_ref.scale_exponents(_words(s), blocks)
    assert (_words(s).transpose(1, 0, 2).reshape(len(v), -1)[:, blocks:] == 127).all()
    full = np.zeros(q.shape)
    full[:, :d] = y
    full = full.reshape(len(v), blocks, 128)
    # A sum of d squares: a lane's 32 in turn, then a tree: at most 32 + 6 + 16 roundings of 2^-24, half of them behind the root;
    # quotient, root, reciprocal and two products: 5 more.  32 in all, so 2^-19 covers them.
    rel = 2.0 ** -19
    top = np.abs(full).max(axis=-1)
    scale = np.ldexp(1.0, exp)
    low, high = top / scale * (1 - rel), top / scale * (1 + rel)
    some = top > 0
    assert (low[some] <= 448).all() and ((high[some] > 224) | (exp[some] == -126)).all() and (exp[~some] == 0).all()
    got = _host(q.float()).reshape(full.shape) * scale[..., None]
    bound = np.maximum(np.abs(full) * (1 + rel) * 2.0 ** -4, scale[..., None] * 2.0 ** -10) + rel * np.abs(full)
    assert (np.abs(got - full) <= bound).all()


@pytest.mark.parametrize("dtype,add_dtype", [("fp32", None), ("fp32", "fp32"), ("fp32", "bf16"), ("bf16", None), ("bf16", "fp32"),
                                             ("bf16", "bf16")])
@pytest.mark.parametrize("rows,d,pad,offset", [
    (1, 1, 0, 0), (1, 1024, 0, 0), (2, 3, 1, 1), (5, 128, 0, 0), (3, 200, 3, 0), (9, 512, 0, 0), (4, 513, 0, 1), (37, 1024, 0, 0), (6, 1025, 7, 2),
    (3, 2048, 0, 0), (2, 2300, 0, 0), (5, 4096, 8, 0), (2, 5000, 1, 0), (3, 8192, 0, 0), (1, 16384, 0, 0), (2, 16385, 0, 0), (1, 32768, 0, 0),
    (1027, 256, 0, 0), (130, 7, 0, 0), (1000, 64, 5, 1), (77, 100, 0, 0), (70, 129, 1, 1), (41, 255, 0, 0), (19, 257, 3, 0)])
def test_rmsnorm(srm, dtype, add_dtype, rows, d, pad, offset):
    rng = np.random.default_rng(rows * 77 + d)
    x = _wide(rng, rows, d, pad, TYPES[dtype], offset, 0.7)
    add = None if add_dtype is None else _wide(rng, rows, d, pad + 1, TYPES[add_dtype], offset, 0.3)
    gain = torch.from_numpy((1 + 0.2 * rng.standard_normal(d)).astype(np.float32)).cuda()
    whole = x._base.clone()
    want = x.clone() if add is None else (x.float() + add.float()).to(x.dtype)
    q, s, untouched = _empty(srm, rows, d)
    print(f"rmsnorm {dtype} + {add_dtype} {rows} x {d} + {pad}, offset {offset}", flush=True)
    srm.rmsnorm_fp8(x, gain, 1e-5, q, s, add=add)
    torch.cuda.synchronize()
    untouched()
    assert torch.equal(x, want)
    x.copy_(whole[offset:].view(rows, d + pad)[:, :d])
    assert torch.equal(x._base, whole), "written between the rows"
    check_norm(want, gain, 1e-5, q, s, d)


def test_rmsnorm_of_empty_and_broken_rows(srm):
    """Rows of zeros have a norm of zeros, zeros behind the row stay zeros; a NaN or an infinity stays in its row."""
    x = torch.randn(5, 700, device="cuda")
    x[1] = 0
    x[2, 17] = float("nan")
    x[3, 600] = float("inf")
    gain = torch.ones(700, device="cuda")
    q, s, untouched = _empty(srm, 5, 700)
    srm.rmsnorm_fp8(x, gain, 1e-6, q, s)
    torch.cuda.synchronize()
    untouched()
    v = q.float()
    assert (v[1] == 0).all() and (s.view(torch.uint8)[:, 1] == 127).all()
    assert v[2, :700].isnan().all() and (v[2, 700:] == 0).all()
    assert v[3, 600].isnan() and (v[3, :600] == 0).all()      # finite / inf
    for r in (0, 4):
        check_norm(x[r:r + 1], gain, 1e-6, q[r:r + 1], s[:, r:r + 1].contiguous(), 700)


def test_a_row_has_the_same_bits_whatever_the_batch(srm):
    rng = np.random.default_rng(11)
    for d in (96, 1024, 3000, 9000):
        x = _wide(rng, 50, d, 0, torch.float32)
        gain = torch.ones(d, device="cuda")
        q, s, _ = _empty(srm, 50, d)
        srm.rmsnorm_fp8(x, gain, 1e-5, q, s)
        for r in (0, 31, 49):
            q1, s1, _ = _empty(srm, 1, d)
            srm.rmsnorm_fp8(x[r:r + 1], gain, 1e-5, q1, s1)
            assert torch.equal(q1.view(torch.uint8)[0], q.view(torch.uint8)[r])
            assert torch.equal(s1.view(torch.uint8)[:, 0], s.view(torch.uint8)[:, r])


# ------------------------------------------------------------------ products
def _matrix(srm, rng, rows, K, scale, whole=False):
    """An fp8 matrix of rows x K and its values: random ones, or whole numbers of a few bits with scales that differ from block to block."""
    kp = -(-K // 128) * 128
    if whole:
        codes = rng.integers(-4, 5, (rows, kp)).astype(np.float64)
        codes[:, K:] = 0
        exp = rng.integers(-2, 3, (rows, kp // 128))
    else:
        x = rng.standard_normal((rows, K)) * scale
        x[:, 5 % K::97] *= 20
        codes, exp = fp8_ref.quantize(x)
    q = torch.from_numpy(codes).float().cuda().to(torch.float8_e4m3fn)
    s = torch.from_numpy(fp8_ref.scale_words(exp)).cuda().view(torch.float8_e8m0fnu)
    return q, s, fp8_ref.dequantize(codes, exp)


SIZES = [(1, 1, 1), (1, 16, 128), (2, 3, 127), (1, 32000, 1024), (15, 100, 129), (16, 16, 512), (17, 64, 513), (33, 257, 640), (37, 4096, 1024),
         (64, 64, 2048), (65, 1000, 1000), (100, 130, 4096), (127, 31, 300), (130, 1024, 128), (256, 256, 256), (257, 260, 384), (300, 512, 1024),
         (513, 1030, 777), (1000, 2000, 128), (1500, 1100, 1152), (2100, 2052, 256), (4099, 516, 640), (77, 8, 16384), (520, 4100, 2100), (9, 5000, 300),
         (3001, 4001, 1000), (2100, 8200, 256), (2060, 8301, 300), (4100, 4700, 1100), (5000, 3000, 100), (2900, 3000, 2100),
         (1450, 4100, 700), (26000, 156, 300), (3755, 872, 1152), (10837, 1721, 256)]


@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear_is_exact_on_whole_numbers(srm, M, N, K):
    """Products and sums of these operands are multiples of 2^-4 below 2^20: any order of fp32 sums holds them exactly.  A misplaced
    element, scale, row or column changes them."""
    rng = np.random.default_rng(M * 7 + N * 3 + K)
    a, sa, av = _matrix(srm, rng, M, K, 1, whole=True)
    w, sw, wv = _matrix(srm, rng, N, K, 1, whole=True)
    print(f"linear_fp8 whole {M} x {N} x {K}", flush=True)
    assert K * 16 * 16 < 1 << 23
    buf = torch.full((M * N + 64,), 7.0, device="cuda")
    out = buf[32:-32].view(M, N)
    srm.linear_fp8(4, a, sa, w, sw, None, out)
    torch.cuda.synchronize()
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all()
    want = torch.from_numpy(av).cuda() @ torch.from_numpy(wv.T.copy()).cuda()
    assert torch.equal(out.double(), want)
    buf = torch.full((M * N + 64,), 7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[32:-32].view(M, N)
    srm.linear_fp8(0, a, sa, w, sw, None, out)
    torch.cuda.synchronize()
    assert (buf[:32] == 7).all() and (buf[-32:] == 7).all() and torch.equal(out, want.bfloat16())


@pytest.mark.parametrize("epilogue", [0, 1, 2, 4])
@pytest.mark.parametrize("M,N,K", SIZES)
def test_linear(srm, M, N, K, epilogue):
    """fp32 sums of K exact products in an order of the hardware's: each of at most Kp + 3 steps (bias and residual among them) loses at
    most 2^-23 of the running magnitude, which the sum of the magnitudes S bounds.  For bf16 outputs the 8-bit matrix instructions add
    eight products in a window that holds 2^-13 of the largest: seven of eight lose at most that, 7 * 2^-13 S in all; and the output
    rounds by 2^-8 on top; the GELU's slope is below 1.13 and its fitted form 1e-6 off."""
    rng = np.random.default_rng(M * 5 + N + K * 3 + epilogue)
    a, sa, av = _matrix(srm, rng, M, K, 1.0)
    w, sw, wv = _matrix(srm, rng, N, K, 1 / np.sqrt(K))
    bias = torch.from_numpy(rng.standard_normal(N).astype(np.float32)).cuda() if (M + N) % 3 else None
    old = torch.from_numpy(rng.standard_normal((M, N)).astype(np.float32)).cuda()
    out = old.clone() if epilogue == 2 else torch.empty((M, N), dtype=torch.float32 if epilogue == 4 else torch.bfloat16, device="cuda")
    print(f"linear_fp8 {M} x {N} x {K} epilogue {epilogue}", flush=True)
    srm.linear_fp8(epilogue, a, sa, w, sw, bias, out)
    torch.cuda.synchronize()
    A, W = torch.from_numpy(av).cuda(), torch.from_numpy(wv.T.copy()).cuda()
    ref, size = A @ W, A.abs() @ W.abs()
    if bias is not None:
        ref, size = ref + bias.double(), size + bias.double().abs()
    if epilogue == 2:
        ref, size = ref + old.double(), size + old.double().abs()
    tol = (a.shape[1] + 3) * 2.0 ** -23 * size
    if epilogue in (0, 1):
        tol = tol + 7 * 2.0 ** -13 * size
    if epilogue == 1:
        ref, tol = ref * torch.special.ndtr(ref), 1.13 * tol + 1e-6
    if epilogue in (0, 1):
        tol = tol + 2.0 ** -8 * ref.abs() * 1.01
    assert ((out.double() - ref).abs() <= tol).all()


def test_linear_at_the_ends_of_the_scales(srm):
    """The largest and smallest scales, a row of zeros, and NaN, which stays in its row or column."""
    M, N, K = 40, 48, 256
    a = torch.ones(M, K, device="cuda").to(torch.float8_e4m3fn)
    w = torch.ones(N, K, device="cuda").to(torch.float8_e4m3fn)
    sa = torch.full((1, M, 4), 127, dtype=torch.uint8, device="cuda")
    sw = torch.full((1, N, 4), 127, dtype=torch.uint8, device="cuda")
    sa[0, 3, :2], sw[0, 5, :2] = 1, 254                       # 2^-126, 2^127
    sa[0, 4, 0], sa[0, 4, 1] = 120, 130                       # blocks of one row
    a.view(torch.uint8)[7] = 0
    a.view(torch.uint8)[9, 130] = 0x7F
    out = torch.empty(M, N, device="cuda")
    srm.linear_fp8(4, a, sa.view(torch.float8_e8m0fnu), w, sw.view(torch.float8_e8m0fnu), None, out)
    fa = torch.exp2(sa[0, :, :2].double() - 127).repeat_interleave(128, 1) * a.double()
    fw = torch.exp2(sw[0, :, :2].double() - 127).repeat_interleave(128, 1) * w.double()
    ref = (fa @ fw.t().contiguous()).float()
    assert out[9].isnan().all() and (out[7] == 0).all()
    keep = [r for r in range(M) if r != 9]
    assert torch.equal(out[keep], ref[keep])


def test_linear_writes_at_any_element(srm):
    """Outputs that lie at no multiple of 16 bytes."""
    rng = np.random.default_rng(3)
    for M, N, K in ((70, 64, 256), (300, 512, 512), (700, 260, 128)):
        a, sa, av = _matrix(srm, rng, M, K, 1, whole=True)
        w, sw, wv = _matrix(srm, rng, N, K, 1, whole=True)
        want = torch.from_numpy(av @ wv.T).cuda()
        for epilogue, dtype in ((4, torch.float32), (2, torch.float32), (0, torch.bfloat16)):
            buf = torch.zeros(M * N + 2, dtype=dtype, device="cuda")
            srm.linear_fp8(epilogue, a, sa, w, sw, None, buf[1:-1].view(M, N))
            assert torch.equal(buf[1:-1].view(M, N), want.to(dtype)) and buf[0] == 0 and buf[-1] == 0


def test_linear_of_more_than_two_gigabytes(srm):
    """Rows and outputs behind 2^31 bytes and elements: the last ones of a tall product against a product of their own."""
    M, N, K = 600_000, 64, 4096
    a, sa = srm.fp8_empty(M, K)
    pattern = torch.randint(0, 0x7E, (1000, K), dtype=torch.uint8, device="cuda") & 0xBF
    a.view(torch.uint8).view(600, 1000, K).copy_(pattern)
    sa.view(torch.uint8).fill_(127)
    rng = np.random.default_rng(8)
    w, sw, _ = _matrix(srm, rng, N, K, 0.02)
    out, part = torch.empty(M, N, device="cuda"), torch.empty(1000, N, device="cuda")
    srm.linear_fp8(4, a, sa, w, sw, None, out)
    srm.linear_fp8(4, a[-1000:], sa[:, -1000:].contiguous(), w, sw, None, part)
    ref = a[-1000:].double() @ torch.from_numpy(_).cuda().t().contiguous()
    size = a[-1000:].double().abs() @ torch.from_numpy(_).cuda().abs().t().contiguous()
    for got in (out[-1000:], part, out[:1000], out[300_000:301_000]):
        assert ((got.double() - ref).abs() <= (K + 3) * 2.0 ** -23 * size).all()


@pytest.mark.parametrize("rows,d", [((1 << 26) + 5, 8), ((1 << 23) + 5, 257)])
def test_more_rows_than_a_dimension_of_a_grid_has_threads_for(srm, rows, d):
    """More work-groups than a row of the grid: the same codes as in a small call."""
    x = torch.zeros(rows, d, device="cuda")
    some = torch.tensor([0, 1, 12345, rows // 8 + 1, rows // 2 - 3, rows // 2, rows - 6, rows - 5, rows - 1], device="cuda")
    few = torch.randn(len(some), d, device="cuda")
    x[some] = few
    (q, s), (qf, sf) = srm.fp8_empty(rows, d), srm.fp8_empty(len(some), d)
    gain = torch.rand(d, device="cuda") + 0.5
    for call in (lambda x, q, s: srm.quantize_fp8(x, q, s), lambda x, q, s: srm.rmsnorm_fp8(x, gain, 1e-5, q, s)):
        q.view(torch.uint8).fill_(0x5A)
        s.view(torch.uint8).fill_(0x5A)
        call(x, q, s)
        call(few, qf, sf)
        assert torch.equal(q.view(torch.uint8)[some], qf.view(torch.uint8)) and torch.equal(s.view(torch.uint8)[:, some], sf.view(torch.uint8))
        q.view(torch.uint8)[some] = 0
        s.view(torch.uint8)[:, some] = 127
        assert int(q.view(torch.int64).amax()) == 0 == int(q.view(torch.int64).amin()) and (s.view(torch.int32) == 0x7F7F7F7F).all()


def test_a_single_row_of_more_columns_than_a_dimension_of_a_grid_has_threads_for(srm):
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("less than 60 GiB of free memory")
    N, K = (1 << 28) + 37, 128
    a, sa = srm.fp8_empty(1, K)
    srm.quantize_fp8(torch.randn(1, K, device="cuda"), a, sa)
    w, sw = srm.fp8_empty(N, K)
    w.view(torch.uint8).zero_()
    sw.view(torch.uint8).fill_(127)
    some = torch.tensor([0, 17, (1 << 26) + 3, (1 << 27) - 1, 1 << 27, (1 << 28) - 1, 1 << 28, N - 1], device="cuda")
    wf, swf = srm.fp8_empty(len(some), K)
    srm.quantize_fp8(torch.randn(len(some), K, device="cuda"), wf, swf)
    w.view(torch.uint8)[some] = wf.view(torch.uint8)
    sw.view(torch.uint8)[:, some] = swf.view(torch.uint8)
    out, few = torch.full((1, N), 7.0, device="cuda"), torch.empty(1, len(some), device="cuda")
    srm.linear_fp8(4, a, sa, w, sw, None, out)
    srm.linear_fp8(4, a, sa, wf, swf, None, few)
    # (another kernel, which adds K's parts in another order)
    size = _values(a, sa).abs() @ _values(wf, swf).abs().t().contiguous()
    assert ((out[:, some] - few).double().abs() <= (K + 3) * 2.0 ** -22 * size).all()
    out[:, some] = 0
    assert (out == 0).all()


# ------------------------------------------------------------------ together
def _block(srm, M, d, ff, rng):
    """A channel mixer in 8 bits: norm, up projection with GELU, quantize, down projection into the residual stream."""
    up, su, _ = _matrix(srm, rng, ff, d, 1 / np.sqrt(d))
    down, sd, _ = _matrix(srm, rng, d, ff, 1 / np.sqrt(ff))
    t = dict(x=torch.randn(M, d, device="cuda"), add=torch.randn(M, d, device="cuda").bfloat16(), gain=torch.rand(d, device="cuda") + 0.5,
             q=srm.fp8_empty(M, d), h=torch.empty(M, ff, dtype=torch.bfloat16, device="cuda"), qh=srm.fp8_empty(M, ff),
             bu=torch.randn(ff, device="cuda"), bd=torch.randn(d, device="cuda"))

    def run():
        srm.rmsnorm_fp8(t["x"], t["gain"], 1e-5, *t["q"], add=t["add"])
        srm.linear_fp8(1, *t["q"], up, su, t["bu"], t["h"])
        srm.quantize_fp8(t["h"], *t["qh"])
        srm.linear_fp8(2, *t["qh"], down, sd, t["bd"], t["x"])
    return t, run, (up, su, down, sd)


def _values(q, s):
    return torch.from_numpy(fp8_ref.dequantize(_host(q.float()), fp8_ref.scale_exponents(_words(s), q.shape[1] // 128))).cuda()


@pytest.mark.parametrize("M,d,ff", [(1, 256, 1024), (37, 512, 2048), (700, 1024, 4096)])
def test_a_channel_mixer_in_8_bits(srm, M, d, ff):
    """Each step against 64 bits on what the step before has left; and the whole against the mixer in 64 bits, whose distance is that of
    two roundings of activations to e4m3 (weights are the same): below 2^-4 of the hidden values' size each, relative to the update."""
    rng = np.random.default_rng(M)
    t, run, (up, su, down, sd) = _block(srm, M, d, ff, rng)
    x0 = t["x"].double() + t["add"].double()
    run()
    torch.cuda.synchronize()
    x1 = x0.float()                                            # the sum as it is stored
    check_norm(x1, t["gain"], 1e-5, *t["q"], d)
    v = _values(*t["q"]) @ _values(up, su).t().contiguous() + t["bu"].double()
    size = _values(*t["q"]).abs() @ _values(up, su).abs().t().contiguous() + t["bu"].double().abs()
    h = v * torch.special.ndtr(v)
    assert ((t["h"].double() - h).abs() <= 1.13 * ((d + 3) * 2.0 ** -23 + 7 * 2.0 ** -13) * size + 1e-6 + 2.0 ** -8 * 1.01 * h.abs()).all()
    want, exp = fp8_ref.quantize(_host(t["h"]))
    np.testing.assert_array_equal(_host(t["qh"][0].float()), want)
    np.testing.assert_array_equal(_words(t["qh"][1]), fp8_ref.scale_words(exp))
    y = _values(*t["qh"]) @ _values(down, sd).t().contiguous() + t["bd"].double()
    size = _values(*t["qh"]).abs() @ _values(down, sd).abs().t().contiguous() + t["bd"].double().abs() + x1.double().abs()
    assert ((t["x"].double() - (x1.double() + y)).abs() <= (ff + 3) * 2.0 ** -23 * size).all()


def test_captured_and_replayed_with_eager_work_between(srm):
    """A graph of the block, replayed on other inputs with the program's eager calls between the replays: the eager bits each time."""
    rng = np.random.default_rng(2)
    t, run, _ = _block(srm, 70, 512, 1024, rng)
    fresh = [(torch.randn(70, 512, device="cuda"), torch.randn(70, 512, device="cuda").bfloat16()) for _ in range(4)]

    def load(i):
        t["x"].copy_(fresh[i][0])
        t["add"].copy_(fresh[i][1])

    eager = []
    for i in range(4):
        load(i)
        run()
        eager.append((t["x"].clone(), t["h"].clone()))
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        run()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    other, other_run, _ = _block(srm, 33, 256, 512, rng)
    for i in (2, 0, 3, 1, 2):
        load(i)
        other_run()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(t["x"], eager[i][0]) and torch.equal(t["h"], eager[i][1])


def test_two_streams_at_once(srm):
    rng = np.random.default_rng(6)
    blocks = [_block(srm, M, 512, 2048, rng) for M in (300, 41)]
    start = [(b[0]["x"].clone(), b[0]["add"].clone()) for b in blocks]
    want = []
    for b in blocks:
        b[1]()
        want.append(b[0]["x"].clone())
    streams = [torch.cuda.Stream() for _ in blocks]
    for _ in range(5):
        for b, (x, add) in zip(blocks, start):
            b[0]["x"].copy_(x)
            b[0]["add"].copy_(add)
        torch.cuda.synchronize()
        for b, st in zip(blocks, streams):
            with torch.cuda.stream(st):
                b[1]()
        torch.cuda.synchronize()
        for b, w in zip(blocks, want):
            assert torch.equal(b[0]["x"], w)


def test_the_stream_argument(srm):
    x = torch.randn(200, 1024, device="cuda")
    a, sa = srm.fp8_empty(200, 1024)
    want = srm.fp8_empty(200, 1024)
    srm.quantize_fp8(x, *want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    srm.quantize_fp8(x, a, sa, stream=st)
    st.synchronize()
    assert torch.equal(a.view(torch.uint8), want[0].view(torch.uint8))
