"""Register budget of the residual norm and the distillation loss, from the compiler's resource report
(CPU): no kernel uses scratch memory, and the rows that stay in registers leave room for the
workgroups that hide their loads."""
import pytest

from tests.test_kernel_resources import _resources


@pytest.mark.parametrize("src,least", [("rms_norm.hip", 40), ("distill.hip", 100)])
def test_no_kernel_spills(src, least):
    rows = _resources(src)
    assert len(rows) >= least
    spills = {k: v["ScratchSize"] for k, v in rows.items() if v.get("ScratchSize", 0) != 0}
    assert not spills, spills
    if src == "distill.hip":  # 13 chunks of 16 bytes a thread: 52 of at most 80 registers
        kept = {k: v["Occupancy"] for k, v in rows.items() if "distill_row_kernel" in k and "ELi13ELi" in k}
        assert len(kept) == 16 and min(kept.values()) >= 6, kept
    else:                     # the gradient's workgroups of 1024 threads: one a CU at least twice over
        most = {k: v["Occupancy"] for k, v in rows.items() if "rms_bwd_kernel" in k}
        assert most and min(most.values()) >= 4, most
