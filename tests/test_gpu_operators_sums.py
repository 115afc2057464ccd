"""Long sums of the operators around the blocks, on inputs whose sums are exact in fp32 when
they are added the way the kernels say."""
import pytest

from paper_2206_04959_amd import binding as B
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d,tokens", [(128, 32), (128, 2048), (128, 4096), (64, 4096), (96, 4096), (80, 1024)])
def test_gain_sums_of_equal_terms_are_exact(d, tokens):
    """Every term of a column's sum is the same number v / 2 (rows of 1/2 and eps = 3/4, so that the
    norm's root is 1 to the last bit; no rotation) and the counts are powers of two, so a tree of
    additions only doubles and rounds nothing.  Adding the last 64 sums in one chain rounded most of its steps
    and missed the exact result in four columns of five."""
    torch = need_gpu()
    print(f"[gains] {tokens} tokens, heads of {d}", flush=True)
    qkv = torch.full((tokens, 3, d), 0.5, device="cuda")
    v = torch.randn(3, d, device="cuda")
    dout = v.expand(tokens, 3, d).contiguous()
    one = torch.ones(d, device="cuda")
    dq, dk = torch.empty(d, device="cuda"), torch.empty(d, device="cuda")
    scratch = torch.empty(B.qk_norm_rope_scratch_elems(tokens, 1, 1, d), device="cuda")
    B.qk_norm_rope_bwd(dout, qkv, one, one, None, torch.empty_like(qkv), dq, dk, scratch, 1, 1, eps=0.75)
    torch.cuda.synchronize()
    assert torch.equal(dq, v[0] * (tokens / 2)) and torch.equal(dk, v[1] * (tokens / 2))


# ---------------------------------------------------------------------------
# Sums of small integers: exact in fp32 in any order, so one lost, doubled or foreign term shows
# ---------------------------------------------------------------------------

def _integers(torch, most, *shape, dtype):
    return torch.randint(-most, most + 1, shape, device="cuda").to(dtype)


def _ids(torch, pattern, tokens, rows):
    if pattern == "same":
        return torch.full((tokens,), rows // 2, device="cuda")
    if pattern == "few":  # long runs, many of them split
        return (torch.rand(tokens, device="cuda") ** 6 * rows).long()
    # runs of 1 .. 99 tokens, spread over the batch: some whole, some split, some just at either
    run = torch.repeat_interleave(torch.arange(rows, device="cuda"), torch.arange(rows, device="cuda") % 99 + 1)
    return run[torch.arange(tokens, device="cuda") * 7919 % tokens]


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,hidden,rows,pattern", [
    (257, 64, 5, "same"), (2048, 520, 300, "few"), (2049, 8, 100, "same"), (2500, 1032, 80, "runs"),
    (5003, 24, 110, "runs"), (17000, 8, 90, "same"), (17000, 520, 700, "few"), (33000, 16, 9, "few"),
    (33000, 8, 3, "same"), (40000, 1000, 900, "runs"), (100001, 64, 2000, "few")])
def test_embedding_gradient_loses_no_token(dtype, tokens, hidden, rows, pattern):
    torch = need_gpu()
    print(f"[embedding bwd] {dtype} {tokens}x{hidden} rows {rows} {pattern}", flush=True)
    torch.manual_seed(tokens)
    ids = _ids(torch, pattern, tokens, rows)
    dy = _integers(torch, 4, tokens, hidden, dtype=getattr(torch, dtype))
    want = torch.zeros(rows + 1, hidden, dtype=torch.float64, device="cuda").index_add_(0, ids, dy.double())[:-1] * 0.5
    base = _integers(torch, 9, rows, hidden, dtype=torch.float32)
    dtable = torch.full((rows, hidden), float("nan"), device="cuda")
    scratch = torch.empty(max(B.embedding_scratch_bytes(tokens, hidden), 1), dtype=torch.uint8, device="cuda")
    B.embedding_bwd(ids, dy, dtable, scratch, scale=0.5)
    torch.cuda.synchronize()
    assert torch.equal(dtable.double(), want)
    dtable.copy_(base)
    B.embedding_bwd(ids, dy, dtable, scratch, scale=0.5, accumulate=True)
    torch.cuda.synchronize()
    assert torch.equal(dtable.double(), base.double() + want)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,q,kv,d,rope,inter", [
    (4200, 12, 12, 64, 64, False), (3001, 24, 6, 128, 128, False), (5000, 9, 3, 96, 48, False),
    (2500, 6, 6, 96, 96, False), (2500, 4, 4, 256, 128, False), (1800, 12, 12, 256, 256, False),
    (3001, 8, 2, 80, 80, True), (4000, 16, 16, 200, 64, True), (4200, 12, 12, 64, 0, False)])
def test_gain_gradient_loses_no_head(dtype, tokens, q, kv, d, rope, inter):
    """Several steps of every workgroup, then the sum over the workgroups.  Rows of +-1/2 with eps =
    3/4 have a norm of 1, and a table of quarter turns moves and negates features: all terms are
    integers and halves."""
    torch = need_gpu()
    print(f"[gains] {dtype} {tokens} tokens {q}+{kv} heads of {d}, rope {rope} inter {inter}", flush=True)
    torch.manual_seed(tokens + d)
    dt = getattr(torch, dtype)
    qkv = (_integers(torch, 1, tokens, q + 2 * kv, d, dtype=torch.float32) >= 0).to(dt) - 0.5
    dout = _integers(torch, 8, tokens, q + 2 * kv, d, dtype=dt)
    one = torch.ones(d, dtype=dt, device="cuda")
    table, kw = None, {}
    back = dout[:, :q + kv].double()
    if rope:
        turn = torch.randint(0, 4, (50, rope // 2), device="cuda")
        table = torch.tensor([[1.0, 0.0], [0.0, 1.0], [-1.0, 0.0], [0.0, -1.0]], device="cuda")[turn].contiguous()
        pos = torch.randint(0, 50, (tokens,), device="cuda")
        kw = dict(positions=pos.int())
        c, s = table[pos][:, None].double().unbind(-1)
        i = torch.arange(rope // 2, device="cuda")
        ia, ib = (2 * i, 2 * i + 1) if inter else (i, i + rope // 2)
        a, b = back[..., ia], back[..., ib]
        back[..., ia], back[..., ib] = a * c + b * s, b * c - a * s
    terms = back * qkv[:, :q + kv].double()
    want = terms[:, :q].sum((0, 1)), terms[:, q:].sum((0, 1))
    base = _integers(torch, 9, 2, d, dtype=torch.float32)
    dq, dk = torch.full((2, d), float("nan"), device="cuda")
    scratch = torch.empty(B.qk_norm_rope_scratch_elems(tokens, q, kv, d), device="cuda")
    dqkv = torch.empty_like(dout)
    for accumulate, add in ((False, torch.zeros_like(base)), (True, base)):
        if accumulate:
            dq, dk = base[0].clone(), base[1].clone()
        B.qk_norm_rope_bwd(dout, qkv, one, one, table, dqkv, dq, dk, scratch, q, kv, interleaved=inter, eps=0.75,
                           accumulate=accumulate, **kw)
        torch.cuda.synchronize()
        assert torch.equal(dq.double(), want[0] + add[0].double())
        assert torch.equal(dk.double(), want[1] + add[1].double())


# What the bf16 shapes take, by the plan of the weight gradient: codes converted by four waves (many stages;
# odd ends; splits), by eight (short and long stages), X restored with 256 x 256, 256 x 192 and 128 x 128
# tiles of eight and of four waves.
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,n_out,n_in", [
    (301, 2056, 4128), (1000, 1024, 8192), (2047, 1000, 4128), (9001, 1400, 1440), (333, 264, 288), (5001, 64, 64),
    (601, 1000, 512), (4101, 1288, 1312), (1025, 6000, 2560), (5001, 1928, 1056), (2001, 5000, 640), (6001, 1600, 1600)])
def test_weight_gradient_loses_no_token(dtype, tokens, n_out, n_in):
    torch = need_gpu()
    print(f"[act8 dw] {dtype} {tokens} tokens, {n_out} x {n_in}", flush=True)
    torch.manual_seed(tokens)
    dt = getattr(torch, dtype)
    x = _integers(torch, 8, tokens, n_in, dtype=dt)  # four significant bits: kept exactly
    dy = _integers(torch, 4, tokens, n_out, dtype=dt)
    q = torch.empty((tokens, n_in), dtype=torch.uint8, device="cuda")
    s = torch.empty((tokens, n_in // 32), dtype=torch.uint8, device="cuda")
    B.act8_save(x, q, s)
    want = torch.mm(dy.double().t().contiguous(), x.double())
    n = B.act8_gemm_dw_scratch_bytes(dt, tokens, n_out, n_in)
    scratch = torch.empty(max(n, 1), dtype=torch.uint8, device="cuda")
    dw = torch.full((n_out, n_in), float("nan"), device="cuda")
    B.act8_gemm_dw(dy, q, s, dw, scratch)
    torch.cuda.synchronize()
    assert torch.equal(dw.double(), want)
    base = _integers(torch, 9, n_out, n_in, dtype=torch.float32)
    dw.copy_(base)
    B.act8_gemm_dw(dy, q, s, dw, scratch, accumulate=True)
    torch.cuda.synchronize()
    assert torch.equal(dw.double(), base.double() + want)
