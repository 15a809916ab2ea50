"""Products of 8-bit rows: operands and outputs that end where their allocations end, and each of the kernels with its shortest loops."""
import numpy as np
import pytest
import torch

import fp8_ref
import gpu_util

pytestmark = pytest.mark.gpu
STORE, GELU, RESIDUAL, LOGITS = 0, 1, 2, 4


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    pkg.lib()
    return pkg


def _last_of_an_allocation(shape, dtype):
    """An uninitialised tensor behind which nothing of its allocation lies (large ones are of whole multiples of 2 MiB)."""
    size = int(np.prod(shape)) * torch.empty(0, dtype=dtype).element_size()
    whole = max(-(-size // (1 << 21)), 8) << 21
    return torch.empty(whole, dtype=torch.uint8, device="cuda")[whole - size:].view(dtype).view(shape)


def _whole_numbers(rng, rows, K):
    """An fp8 matrix of whole numbers from -4 to 4 with scales from 2^-2 to 2^2 that differ from block to block, and its values."""
    kp = -(-K // 128) * 128
    codes = rng.integers(-4, 5, (rows, kp)).astype(np.float64)
    codes[:, K:] = 0
    exp = rng.integers(-2, 3, (rows, kp // 128))
    words = fp8_ref.scale_words(exp)
    q, s = _last_of_an_allocation((rows, kp), torch.float8_e4m3fn), _last_of_an_allocation(words.shape, torch.uint8)
    q.copy_(torch.from_numpy(codes).float().cuda().to(torch.float8_e4m3fn))
    s.copy_(torch.from_numpy(words).cuda())
    return q, s.view(torch.float8_e8m0fnu), torch.from_numpy(fp8_ref.dequantize(codes, exp)).cuda()


def check_product(srm, M, N, K, epilogue, around=lambda call: call()):
    """Products and sums of these operands are multiples of 2^-4 below 2^20, which fp32 sums hold in any order; the GELU is within
    6.5e-7, and bf16 rounds by 2^-8."""
    rng = np.random.default_rng(M * 7 + N * 3 + K + epilogue)
    assert K * 16 * 16 < 1 << 23
    a, sa, av = _whole_numbers(rng, M, K)
    w, sw, wv = _whole_numbers(rng, N, K)
    bias = _last_of_an_allocation((N,), torch.float32)
    bias.copy_(torch.from_numpy(rng.integers(-64, 65, N).astype(np.float32)))
    out = _last_of_an_allocation((M, N), torch.float32 if epilogue in (RESIDUAL, LOGITS) else torch.bfloat16)
    old = torch.from_numpy(rng.integers(-64, 65, (M, N)).astype(np.float32)).cuda() if epilogue == RESIDUAL else 0.0
    print(f"linear_fp8 {M} x {N} x {K} epilogue {epilogue}", flush=True)

    def call():
        out.copy_(old) if epilogue == RESIDUAL else out.fill_(7.0)
        srm.linear_fp8(epilogue, a, sa, w, sw, bias, out)

    result = around(call)
    torch.cuda.synchronize()
    want = av @ wv.t().contiguous() + bias.double() + (old.double() if epilogue == RESIDUAL else 0.0)
    if epilogue == GELU:
        want = want * torch.special.ndtr(want)
        assert ((out.double() - want).abs() <= 6.5e-7 + 2.0 ** -8 * want.abs()).all()
    else:
        assert torch.equal(out, want.to(out.dtype))
    return result


@pytest.mark.parametrize("M,N,K,epilogue", [
    (1, 1, 1, STORE), (17, 33, 129, LOGITS), (9, 5000, 300, STORE), (700, 1000, 300, RESIDUAL), (1100, 1028, 300, GELU), (3755, 872, 300, STORE),
    (2900, 3000, 256, STORE), (2817, 2817, 384, GELU), (3001, 4001, 1000, STORE), (5000, 5000, 300, LOGITS)])
def test_operands_at_the_end_of_an_allocation(srm, M, N, K, epilogue):
    """Rows of a last tile that do not exist lie behind the allocations: none of them is read or written."""
    check_product(srm, M, N, K, epilogue)


# The kernel that each size is there for, on 256 compute units: every kernel with either kind of output, and of the persistent one
# the fewest blocks of K (two, with one and with several tiles a work-group), three, four (a whole word of scales), five and eight of them.
KERNELS = [
    (33, 257, 640, STORE, "slices_kernel<1, 1, 2"), (9, 5000, 300, STORE, "slices_kernel<1, 2, 1"), (37, 4096, 300, GELU, "slices_kernel<2, 2, 1"),
    (700, 1000, 300, STORE, "slices_kernel<4, 4, 1"), (1100, 1028, 300, STORE, "tile_kernel<64, 64, 2, 2, 4"), (2100, 1030, 300, STORE, "tile_kernel<64, 64, 2, 2, 2"),
    (3755, 872, 300, STORE, "tile_kernel<64, 128, 2, 2, 2"), (3001, 2060, 128, STORE, "tile_kernel<128, 128, 2, 4, 2"),
    (10837, 1721, 256, GELU, "tile_kernel<128, 128, 2, 4, 2"),
    (2900, 3000, 256, STORE, "persist_kernel<"), (8100, 8190, 256, GELU, "persist_kernel<"), (8190, 8100, 200, STORE, "persist_kernel<"),
    (5000, 5000, 300, STORE, "persist_kernel<"), (8100, 5000, 500, STORE, "persist_kernel<"), (4200, 4700, 640, GELU, "persist_kernel<"),
    (6000, 4001, 1024, STORE, "persist_kernel<"),
    (33, 257, 640, RESIDUAL, "slices_kernel<1, 1, 2"), (9, 5000, 300, LOGITS, "slices_kernel<1, 2, 1"), (37, 4096, 300, LOGITS, "slices_kernel<2, 2, 1"),
    (700, 1000, 300, RESIDUAL, "slices_kernel<4, 4, 1"), (1100, 1028, 300, LOGITS, "tile_kernel<64, 64, 2, 2, 4"),
    (2100, 1030, 300, RESIDUAL, "tile_kernel<64, 64, 2, 2, 2"), (3755, 872, 300, LOGITS, "tile_kernel<64, 128, 2, 2, 2"),
    (2900, 3000, 256, RESIDUAL, "tile_kernel<64, 64, 2, 2, 2"), (2900, 3000, 256, LOGITS, "tile_kernel<64, 128, 2, 2, 2"),
    (26000, 156, 300, LOGITS, "tile_kernel<128, 64, 2, 2, 2"), (3001, 2500, 300, RESIDUAL, "tile_kernel<128, 128, 2, 4, 2"),
    (3001, 4001, 2000, RESIDUAL, "tile_kernel<128, 128, 2, 2, 2"), (5000, 5000, 300, LOGITS, "tile_kernel<128, 128, 2, 2, 2")]


@pytest.mark.parametrize("M,N,K,epilogue,kernel", KERNELS)
def test_each_kernel(srm, M, N, K, epilogue, kernel):
    """A change of the rule that sends a size elsewhere leaves a kernel, or the form of it that the size is there for, without a test."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 256:
        pytest.skip("the table is that of 256 compute units")
    events = check_product(srm, M, N, K, epilogue, around=lambda call: gpu_util.kernel_events("gemm_fp8", call))
    assert [kernel in e.name for e in events] == [True], [e.name for e in events]
