"""Register budget of the kernels around the blocks, from the compiler's resource report (CPU): no
kernel uses scratch memory, the 256-wide weight-gradient tiles fit two waves per SIMD,
and the gradient of the query/key norm has the waves that its grid is sized for."""
import pytest

from tests.test_kernel_resources import _resources


@pytest.mark.parametrize("src,least", [("embedding.hip", 14), ("qk_norm_rope.hip", 50), ("act8.hip", 12)])
def test_no_kernel_spills(src, least):
    rows = _resources(src)
    assert len(rows) >= least
    spills = {k: v["ScratchSize"] for k, v in rows.items() if v.get("ScratchSize", 0) != 0}
    assert not spills, spills
    if src == "act8.hip":
        tiles = {k: v["Occupancy"] for k, v in rows.items() if "act8_dw_kernelILi256E" in k}
        assert len(tiles) == 2 and min(tiles.values()) >= 2, tiles
    if src == "qk_norm_rope.hip":  # workgroups of four waves: as many a CU as waves per SIMD
        two = {k: v["Occupancy"] for k, v in rows.items() if "qk_bwd_kernel" in k and "ELi2ELi" in k}
        three = {k: v["Occupancy"] for k, v in rows.items() if "qk_bwd_kernel" in k and "ELi3ELi" in k}
        assert two and min(two.values()) >= 4, two
        assert three and min(three.values()) >= 3, three
