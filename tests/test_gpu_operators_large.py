"""Calls of the operators around the blocks that take more workgroups than one launch can
have: its threads are counted in 32 bits, so 2^24 - 1 workgroups of 256."""
import pytest

from paper_2206_04959_amd import binding as B
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens", [5, 3000])  # in one launch, sorted
def test_embedding_gradient_clears_many_rows(tokens):
    torch = need_gpu()
    rows, h = (1 << 28) + 100, 8  # 16 rows a workgroup: 2^24 + 7
    print(f"[embedding bwd] {tokens} tokens on {rows} rows", flush=True)
    ids = torch.arange(tokens, device="cuda") * 3
    ids[-2:] = torch.tensor([rows - 1, rows - 17])
    dy = torch.randn(tokens, h, device="cuda")
    dtable = torch.full((rows, h), float("nan"), device="cuda")
    scratch = torch.empty(max(B.embedding_scratch_bytes(tokens, h), 1), dtype=torch.uint8, device="cuda")
    B.embedding_bwd(ids, dy, dtable, scratch)
    torch.cuda.synchronize()
    assert torch.equal(dtable[ids], dy)
    dtable[ids] = 0
    assert not dtable.any()  # (NaN counts as true: every other row was cleared)
