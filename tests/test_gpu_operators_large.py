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


@pytest.mark.parametrize("seq", [None, 7, (1 << 20) + 11])  # positions given, short sequences, one in two launches
def test_qk_norm_of_many_small_heads(seq):
    torch = need_gpu()
    T, q, d = (1 << 20) + 2005, 511, 16  # 32 heads a workgroup: 2^24 + 32081 with the keys'
    print(f"[qk fwd] {T} tokens of {q} + 1 heads of {d}, seq {seq}", flush=True)
    row = torch.randn(1, q + 2, d, device="cuda").bfloat16()
    qkv = row.repeat(T, 1, 1)
    one = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    table = torch.empty(((1 << 20) + 11, d // 2, 2), device="cuda")
    B.rope_table(table)
    n = 1 << 20  # one launch holds n - 1 tokens
    at = torch.tensor([0, 1, T // 2, n - 3, n - 2, n - 1, n, n + 5, n + 20, T - 1], device="cuda")
    if seq is None:
        every = (torch.arange(T, device="cuda") * 13 % 1000).int()
        where, kw = every[at], dict(positions=every)
    else:
        where, kw = (at % seq).int(), dict(seq_len=seq)
    B.qk_norm_rope_fwd(qkv, one, one, table, qkv, q, 1, **kw)
    few = row.repeat(at.numel(), 1, 1)
    B.qk_norm_rope_fwd(few, one, one, table, few, q, 1, positions=where)
    torch.cuda.synchronize()
    assert torch.equal(qkv[at], few)
    if seq == 7:  # all tokens at one position have the same rows
        whole = T // 7 * 7
        assert torch.equal(qkv[:whole].view(-1, 7, q + 2, d), qkv[:7].expand(whole // 7, 7, q + 2, d))
