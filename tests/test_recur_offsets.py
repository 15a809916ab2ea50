"""Offsets of packed sequences as a program may hold them: other types than int32, values that do not fit, no rows at all (no GPU)."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def srm():
    import paper_2605_08696_amd as pkg
    from paper_2605_08696_amd import build as b
    if b.is_stale():
        b.build_lib()
    pkg.lib()
    return pkg


def _calls(srm, offsets):
    bf, n = torch.bfloat16, 2
    d_off = torch.zeros(n, dtype=torch.int32)
    x, w, out = torch.zeros(5, 24, dtype=bf), torch.zeros(24, 4), torch.zeros(5, 24, dtype=bf)
    yield lambda: srm.causal_conv(x, w, None, offsets, d_off, out)
    yield lambda: srm.selective_scan(x, torch.zeros(5, 2), torch.zeros(2), offsets, d_off, torch.zeros(5, 8, dtype=bf))
    yield lambda: srm.selective_scan_workspace_bytes(srm.SRM_BF16, offsets, 2, 4, 8)


@pytest.mark.parametrize("offsets", [np.array([0, 2 ** 32 + 5]), np.array([2 ** 32, 5]), torch.tensor([0, 2 ** 33 + 1]), np.array([0.0, 4.5]),
                                     np.array([0, 2 ** 31], dtype=np.uint32), [0, 2.5], np.array([0.0, np.nan])])
def test_values_that_are_no_int32_are_refused(srm, offsets):
    for call in _calls(srm, offsets):
        with pytest.raises(ValueError, match="whole"):
            call()


@pytest.mark.parametrize("offsets", [[0, 5], (0, 5), np.array([0, 5]), torch.tensor([0, 5]), np.array([0, 9, 5, 9], dtype=np.int32)[::2], np.array([0.0, 5.0])])
def test_other_holders_of_whole_values_are_taken(srm, offsets):
    conv, scan, need = _calls(srm, offsets)
    for call in (conv, scan):
        with pytest.raises(ValueError, match="CUDA"):          # all that is wrong is the tensors' place
            call()
    assert need() == 0


def test_plans_of_ragged_prompts_refuse_them_too(srm):
    with pytest.raises(ValueError, match="whole"):
        srm.prefill_ragged_plan(None, np.array([0, 2 ** 32 + 5]), 0)


def test_no_rows_at_all_are_no_work(srm, monkeypatch):
    """Arrays of no rows lie nowhere: not refused, nothing launched; what is wrong with the call otherwise still is."""
    from paper_2605_08696_amd import binding
    codes = []
    monkeypatch.setattr(binding, "_launch", lambda fn, args, first, others, stream: codes.append(fn(*args, None)))
    bf, off, d_off = torch.bfloat16, np.zeros(3, dtype=np.int32), torch.zeros(3, dtype=torch.int32)
    x, w = torch.zeros(0, 24, dtype=bf), torch.zeros(24, 4)
    assert x.data_ptr() == 0
    srm.causal_conv(x, w, None, off, d_off, torch.zeros(0, 24, dtype=bf))
    srm.selective_scan(x, torch.zeros(0, 2), torch.zeros(2), off, d_off, torch.zeros(0, 8, dtype=bf), state=torch.zeros(2, 2, 4, 8))
    assert codes == [0, 0]
    with pytest.raises(ValueError, match="rows"):
        srm.causal_conv(x, w, None, [0, 0, 1], d_off, torch.zeros(0, 24, dtype=bf))
    with pytest.raises(ValueError, match="weight"):
        srm.causal_conv(x, w[:-1], None, off, d_off, torch.zeros(0, 24, dtype=bf))
