"""What the compiler made of the kernels of the selective recurrence, its convolution and the scores of tokens: the metadata of their code
object, the third in the library (no GPU)."""
import os

import pytest

from paper_2605_08696_amd import build
from test_operator_resources import MAGIC, _kernels_of


@pytest.fixture(scope="module")
def kernels():
    if not os.path.exists(build.LIB):
        build.build_lib()
    data = open(build.LIB, "rb").read()
    at = -1
    for _ in range(3):
        at = data.index(MAGIC, at + 1)
    return _kernels_of(data, at)


def test_the_third_code_object_holds_the_operators(kernels):
    for name in ("causal_conv_kernel", "selective_scan_kernel", "selective_scan_mfma_kernel", "selective_scan_join_kernel", "selective_step_kernel",
                 "token_logprobs_kernel"):
        assert any(name in n for n in kernels), name


def test_what_spills_are_segments_of_rows_that_do_not_lie_whole_and_of_fp32(kernels):
    """A few registers that live across a segment's sequences, outside the loop over blocks."""
    spilled = {n: (q[".vgpr_spill_count"], q[".private_segment_fixed_size"]) for n, q in kernels.items()
               if q[".vgpr_spill_count"] or q[".private_segment_fixed_size"]}
    allowed = {n: v for n, v in spilled.items() if ("selective_scan_mfma_kernel" in n and "ELi2ELb0E" in n) or ("selective_scan_kernel" in n and "ELi2E" in n)}
    assert spilled == allowed and all(v[0] <= 16 and v[1] <= 64 for v in allowed.values()), spilled


def test_scans_fit_the_work_groups_that_their_rules_count_on(kernels):
    """Three work-groups of four wavefronts on a CU for whole rows of states up to 128, in registers and LDS."""
    seen = 0
    for n, q in kernels.items():
        if "selective_scan_mfma_kernelILi128E" in n and "ELb1E" in n:
            seen += 1
            assert q[".vgpr_count"] <= 168 and q[".group_segment_fixed_size"] * 3 <= 160 * 1024, n
    assert seen == 3
