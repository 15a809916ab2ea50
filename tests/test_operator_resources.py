"""What the compiler made of the kernels of 8-bit rows, their products and sampling by request: the metadata of their own code object,
which follows that of the generation kernels in the library (no GPU)."""
import os
import struct

import pytest

from paper_2605_08696_amd import build

msgpack = pytest.importorskip("msgpack")
MAGIC = b"__CLANG_OFFLOAD_BUNDLE__"


def _kernels_of(data, base):
    (n,) = struct.unpack_from("<Q", data, base + 24)
    at = base + 32
    for _ in range(n):
        off, size, length = struct.unpack_from("<QQQ", data, at)
        triple = data[at + 24:at + 24 + length]
        at += 24 + length
        if b"gfx950" not in triple:
            continue
        elf = data[base + off:base + off + size]
        (table,) = struct.unpack_from("<Q", elf, 40)
        entry, count = struct.unpack_from("<HH", elf, 58)
        for k in range(count):
            (kind,) = struct.unpack_from("<I", elf, table + k * entry + 4)
            if kind == 7:                                        # SHT_NOTE
                (note,) = struct.unpack_from("<Q", elf, table + k * entry + 24)
                name_len, desc_len, _ = struct.unpack_from("<III", elf, note)
                desc = note + 12 + ((name_len + 3) & ~3)
                return {q[".name"]: q for q in msgpack.unpackb(elf[desc:desc + desc_len])["amdhsa.kernels"]}
    raise AssertionError("no gfx950 code object with metadata in a bundle")


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(build.LIB):
        build.build_lib()
    data = open(build.LIB, "rb").read()
    first = data.index(MAGIC)
    return _kernels_of(data, data.index(MAGIC, first + 1))


def test_the_second_code_object_holds_the_operators(kernels):
    for name in ("quantize_fp8_kernel", "rmsnorm_fp8_kernel", "gemm_fp8_tile_kernel", "gemm_fp8_slices_kernel", "gemm_fp8_persist_kernel",
                 "sample_rows_kernel"):
        assert any(name in n for n in kernels), name


def test_no_operator_spills(kernels):
    """sample_rows_kernel of bf16 logits apart: three registers that live across its passes lie in scratch memory, outside their loops."""
    spilled = {n: (q[".vgpr_spill_count"], q[".private_segment_fixed_size"]) for n, q in kernels.items()
               if q[".vgpr_spill_count"] or q[".private_segment_fixed_size"]}
    samplers = {n: v for n, v in spilled.items() if "sample_rows_kernelIDF16b" in n}
    assert spilled == samplers and all(v[0] <= 4 and v[1] <= 16 for v in samplers.values()), spilled


def test_operators_fit_the_work_groups_that_their_rules_count_on(kernels):
    """Two work-groups of a 128x128 tile on a CU, two of a sampler of 512 threads; one of a persistent 256x256 tile."""
    for n, q in kernels.items():
        registers = q[".vgpr_count"]                             # accumulation registers included
        waves = q[".max_flat_workgroup_size"] // 64
        if "gemm_fp8_tile_kernel" in n:
            assert registers * waves <= 1024, n                  # a SIMD's 512 registers for a quarter of two work-groups' wavefronts
        if "sample_rows_kernel" in n:
            assert registers <= 128 and q[".group_segment_fixed_size"] * (2 if waves == 8 else 1) <= 160 * 1024, n
        if "gemm_fp8_persist_kernel" in n:
            assert registers <= 256, n
