"""Forms of the operators around the blocks that their other tests do not reach: the query/key
kernels' lane layouts, sums over several steps of a workgroup, and the sorted embedding gradient and
the weight gradient from restored values under capture, on two streams and with shared scratch."""
import pytest

from paper_2206_04959_amd import binding as B
from tests import test_gpu_operators as G
from tests import test_gpu_operators_use as U
from tests.gpu_util import need_gpu

pytestmark = pytest.mark.gpu


# Lanes, chunks and how pairs meet: (8, 2, in a lane), (16, 2, in a lane), (16, 2, 8 lanes apart),
# (4, 2, neighbours), (32, 1, neighbours), and those with a last workgroup that is full or has one head.
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,q,kv,d,rope,inter,positions", [
    (67, 5, 5, 128, 128, False, True), (64, 4, 4, 128, 128, False, False), (1, 32, 8, 128, 128, False, True),
    (35, 7, 3, 256, 256, False, True), (33, 3, 1, 256, 128, False, False), (16, 8, 8, 256, 128, False, True),
    (65, 3, 2, 64, 64, True, True), (129, 1, 1, 64, 32, True, False), (41, 3, 2, 200, 64, True, True),
    (9, 4, 4, 248, 240, True, False), (300, 12, 12, 128, 64, False, True), (30, 4, 2, 96, 32, False, True)])
def test_qk_lane_layouts(dtype, tokens, q, kv, d, rope, inter, positions):
    G.test_qk_norm_rope(dtype, tokens, q, kv, d, rope, inter, positions)


# Queries of more heads than the gradient's workgroups hold at once: each takes several steps.
@pytest.mark.parametrize("tokens,q,kv,d,rope", [(4200, 12, 12, 64, 64), (1500, 24, 6, 128, 128), (2100, 12, 12, 96, 96)])
def test_qk_gradient_of_several_steps(tokens, q, kv, d, rope):
    G.test_qk_norm_rope("bf16", tokens, q, kv, d, rope, False, True)


class _Large(U._All):
    """As _All, with the embedding gradient sorted (runs that are split, so parts are joined) and
    the weight gradient from restored values in several splits: both use their scratch."""

    def __init__(self, torch, seed, tokens=5000, rows=150):
        self.n_out, self.n_in = 1928, 1056
        super().__init__(torch, seed, tokens=tokens, rows=rows)
        new = lambda *s, dtype=torch.bfloat16: torch.empty(s, dtype=dtype, device="cuda")  # noqa: E731
        self.x2, self.dy2 = new(tokens, self.n_in), new(tokens, self.n_out)
        self.q2, self.scales2 = new(tokens, self.n_in, dtype=torch.uint8), new(tokens, self.n_in // 32, dtype=torch.uint8)
        self.dw2 = new(self.n_out, self.n_in, dtype=torch.float32)
        n = B.act8_gemm_dw_scratch_bytes(torch.bfloat16, tokens, self.n_out, self.n_in)
        self.s4 = new(n, dtype=torch.uint8)
        assert self.s1.numel() > 0 and n > 2 * tokens * self.n_in  # the values, and sums of splits
        self.fresh()

    def fresh(self):
        super().fresh()
        for t in ("x2", "dy2"):
            if hasattr(self, t):
                t = getattr(self, t)
                t.copy_(self.torch.randn(t.shape, generator=self.g, device="cuda"))

    def run(self, stream=None):
        super().run(stream)
        B.act8_save(self.x2, self.q2, self.scales2, stream=stream)
        B.act8_gemm_dw(self.dy2, self.q2, self.scales2, self.dw2, self.s4, stream=stream)

    def outputs(self):
        return {**super().outputs(), "q2": self.q2.clone(), "scales2": self.scales2.clone(), "dw2": self.dw2.clone()}


def _once(torch, p):
    p.run()
    torch.cuda.synchronize()
    out = p.outputs()
    # the sums that scratch is used for, against 64 bits: at most T terms, in any order
    ids = p.ids.clamp(max=p.rows)
    want = torch.zeros(p.rows + 1, p.H, dtype=torch.float64, device="cuda").index_add_(0, ids, 2.0 * p.dy.double())
    mag = torch.zeros_like(want).index_add_(0, ids, 2.0 * p.dy.double().abs())
    assert ((out["dtable"].double() - want[:-1]).abs() <= p.T * G.U * mag[:-1]).all()
    return out


def test_two_streams_with_scratch_in_use():
    torch = need_gpu()
    a, b = _Large(torch, 1), _Large(torch, 2, tokens=4500, rows=90)
    want = []
    for p in (a, b):
        want.append(_once(torch, p))
        p.clear()
    torch.cuda.synchronize()
    s = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        a.run(s[0])
        b.run(s[1])
    torch.cuda.synchronize()
    U._same(a.outputs(), want[0])
    U._same(b.outputs(), want[1])


def test_capture_and_replay_with_scratch_in_use():
    """The list of split runs begins anew in every replay, with any number of them."""
    torch = need_gpu()
    p = _Large(torch, 3)
    p.run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.run()
    for i in range(4):
        p.fresh()
        if i == 1:
            p.ids.fill_(7)  # one run
        if i == 2:
            p.ids.copy_(torch.arange(p.T, device="cuda") % p.rows)  # none over 34 tokens
        want = _once(torch, p)
        p.clear()
        for t in (p.s1, p.s4):
            t.fill_(0xA5)  # nothing is taken from one call for the next
        graph.replay()
        if i % 2:
            graph.replay()
        torch.cuda.synchronize()
        U._same(p.outputs(), want)


def test_graphs_that_share_scratch_in_use():
    torch = need_gpu()
    a, b = _Large(torch, 4), _Large(torch, 5, tokens=4500, rows=60)
    assert b.s1.numel() <= a.s1.numel() and b.s4.numel() <= a.s4.numel()
    b.s1, b.s2, b.s4 = a.s1, a.s2, a.s4
    want, graphs = [], []
    for p in (a, b):
        want.append(_once(torch, p))
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            p.run()
        graphs.append(graph)
    for _ in range(3):
        a.clear(), b.clear()
        for graph in graphs:
            graph.replay()
        torch.cuda.synchronize()
        U._same(a.outputs(), want[0])
        U._same(b.outputs(), want[1])


# ---------------------------------------------------------------------------
# Calls in place, and without g
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,q,kv,d,rope", [(1, 4, 4, 128, 128), (333, 24, 6, 128, 128), (70, 3, 3, 80, 80)])
def test_qk_in_place_from_views(tokens, q, kv, d, rope):
    """Rows in the middle of larger buffers: the call in place touches its own tokens only."""
    torch = need_gpu()
    torch.manual_seed(tokens)
    whole = torch.randn(tokens + 5, q + 2 * kv, d, device="cuda").bfloat16()
    grads = torch.randn(tokens + 5, q + 2 * kv, d, device="cuda").bfloat16()
    one = torch.ones(d, dtype=torch.bfloat16, device="cuda")
    table = torch.empty((500, rope // 2, 2), device="cuda")
    B.rope_table(table)
    dg = [torch.empty(d, device="cuda") for _ in range(4)]
    scratch = torch.empty(B.qk_norm_rope_scratch_elems(tokens, q, kv, d), device="cuda")
    raw, dout = whole[2:tokens + 2].clone(), grads[2:tokens + 2].clone()
    out, dqkv = torch.empty_like(raw), torch.empty_like(raw)
    B.qk_norm_rope_fwd(raw, one, one, table, out, q, kv, seq_len=500)
    B.qk_norm_rope_bwd(dout, raw, one, one, table, dqkv, dg[0], dg[1], scratch, q, kv, seq_len=500)
    before = whole.clone(), grads.clone()
    view, gview = whole[2:tokens + 2], grads[2:tokens + 2]
    B.qk_norm_rope_bwd(gview, view, one, one, table, gview, dg[2], dg[3], scratch, q, kv, seq_len=500)
    B.qk_norm_rope_fwd(view, one, one, table, view, q, kv, seq_len=500)
    torch.cuda.synchronize()
    assert torch.equal(view, out) and torch.equal(gview, dqkv)
    assert torch.equal(dg[0], dg[2]) and torch.equal(dg[1], dg[3])
    for now, then in zip((whole, grads), before):
        assert torch.equal(now[:2], then[:2]) and torch.equal(now[tokens + 2:], then[tokens + 2:])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_gelu_gradient_without_its_output(dtype):
    torch = need_gpu()
    torch.manual_seed(3)
    x = (torch.randn(333, 352, device="cuda") * 3).to(getattr(torch, dtype))
    q, s = torch.empty((333, 352), dtype=torch.uint8, device="cuda"), torch.empty((333, 11), dtype=torch.uint8, device="cuda")
    B.act8_save(x, q, s)
    dg = torch.randn(333, 352, device="cuda").to(x.dtype)
    du, g, alone = torch.empty_like(dg), torch.empty_like(dg), torch.empty_like(dg)
    B.act8_gelu_bwd(dg, q, s, du, g)
    B.act8_gelu_bwd(dg, q, s, alone)
    B.act8_gelu_bwd(dg, q, s, dg)
    torch.cuda.synchronize()
    assert torch.equal(du, alone) and torch.equal(du, dg)


# ---------------------------------------------------------------------------
# Values that are not finite, in the arrays and behind them
# ---------------------------------------------------------------------------

def _before(torch, t, bad):
    """t at the start of an allocation whose rest holds `bad`."""
    whole = torch.full((t.numel() + 4096 * t.shape[-1],), bad, dtype=t.dtype, device="cuda")
    out = whole[:t.numel()].view(t.shape)
    out.copy_(t)
    return out


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,n_out,n_in", [(301, 2056, 4128), (333, 264, 288), (601, 1000, 512), (1025, 6000, 2560),
                                               (5001, 1928, 1056), (2001, 5000, 640), (6001, 1600, 1600), (1, 8, 32)])
def test_weight_gradient_keeps_non_finite_values_apart(dtype, tokens, n_out, n_in):
    """NaN behind the last token changes nothing; a NaN or an infinity of dy is in its output's row of dw,
    a NaN of X in its input's column, and every other element keeps its bits."""
    torch = need_gpu()
    print(f"[act8 dw] {dtype} {tokens} tokens, {n_out} x {n_in}", flush=True)
    torch.manual_seed(tokens)
    dt = getattr(torch, dtype)
    x, dy = torch.randn(tokens, n_in, device="cuda").to(dt), torch.randn(tokens, n_out, device="cuda").to(dt)
    scratch = torch.empty(max(B.act8_gemm_dw_scratch_bytes(dt, tokens, n_out, n_in), 1), dtype=torch.uint8, device="cuda")

    def run(dy, x, behind):
        q = torch.empty((tokens, n_in), dtype=torch.uint8, device="cuda")
        s = torch.empty((tokens, n_in // 32), dtype=torch.uint8, device="cuda")
        B.act8_save(x, q, s)
        if behind:
            dy, q, s = _before(torch, dy, float("nan")), _before(torch, q, 0x7F), _before(torch, s, 200)
        scratch.fill_(0xFF)
        dw = torch.empty((n_out, n_in), device="cuda")
        B.act8_gemm_dw(dy, q, s, dw, scratch)
        torch.cuda.synchronize()
        return dw

    clean = run(dy, x, False)
    assert torch.isfinite(clean).all() and torch.equal(run(dy, x, True), clean)
    dy[0, n_out - 1], dy[tokens // 2, n_out // 2], x[tokens - 1, n_in - 1] = float("nan"), float("inf"), float("nan")
    got = run(dy, x, True)
    rows, cols = [n_out - 1, n_out // 2], n_in - 1
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[rows] = True
    bad[:, cols] = True
    assert not torch.isfinite(got[bad]).any() and torch.equal(got[~bad], clean[~bad])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,hidden,rows", [(70, 72, 9), (2048, 8, 40), (5003, 520, 60)])
def test_embedding_keeps_non_finite_values_apart(dtype, tokens, hidden, rows):
    torch = need_gpu()
    print(f"[embedding] {dtype} {tokens}x{hidden} rows {rows}", flush=True)
    torch.manual_seed(tokens)
    dt = getattr(torch, dtype)
    ids = (torch.rand(tokens, device="cuda") ** 2 * (rows + 3)).long()
    ids[tokens // 3] = -1
    dy = _before(torch, torch.randn(tokens, hidden, device="cuda").to(dt), float("nan"))
    scratch = torch.empty(max(B.embedding_scratch_bytes(tokens, hidden), 1), dtype=torch.uint8, device="cuda")

    def run():
        d = torch.full((rows, hidden), float("nan"), device="cuda")
        scratch.fill_(0xFF)
        B.embedding_bwd(ids, dy, d, scratch)
        torch.cuda.synchronize()
        return d

    clean = run()
    assert torch.isfinite(clean).all()
    mine = ((ids >= 0) & (ids < rows)).nonzero()[:, 0]
    t = int(mine[mine.numel() // 2])
    dy[t, 3], dy[tokens // 3] = float("inf"), float("nan")  # one that counts, one of padding
    got = run()
    bad = torch.zeros_like(got, dtype=torch.bool)
    bad[ids[t], 3] = True
    assert torch.isinf(got[bad]).all() and torch.equal(got[~bad], clean[~bad])
    table = torch.randn(rows, hidden, device="cuda").to(dt)
    table[1, 2] = float("nan")
    y = torch.empty((tokens, hidden), dtype=dt, device="cuda")
    B.embedding_fwd(ids, table, y)
    torch.cuda.synchronize()
    want = torch.zeros_like(y)
    want[:, 2] = (ids == 1).to(dt)
    assert torch.equal(torch.isnan(y), want.bool()) and not y[(ids < 0) | (ids >= rows)].any()


# ---------------------------------------------------------------------------
# The widest rows and the most heads that the entry points take
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [70, 2100])
def test_embedding_of_the_widest_rows(tokens):
    torch = need_gpu()
    h, rows = 1 << 20, 6
    print(f"[embedding] {tokens}x{h}", flush=True)
    torch.manual_seed(tokens)
    ids = torch.randint(0, rows - 1, (tokens,), device="cuda")
    dy = torch.randint(-4, 5, (tokens, h), device="cuda", dtype=torch.int8).bfloat16()
    dtable = torch.full((rows, h), float("nan"), device="cuda")
    scratch = torch.empty(max(B.embedding_scratch_bytes(tokens, h), 1), dtype=torch.uint8, device="cuda")
    B.embedding_bwd(ids, dy, dtable, scratch)
    torch.cuda.synchronize()
    for r in range(rows):
        assert torch.equal(dtable[r], dy[ids == r].float().sum(0))
    table = dtable.bfloat16()
    y = torch.empty_like(dy)
    B.embedding_fwd(ids, table, y)
    torch.cuda.synchronize()
    assert torch.equal(y, table[ids])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens,n_out,n_in", [(3, 8, 1 << 20), (3, 1 << 20, 32), (130, 264, 1 << 18), (130, 1 << 18, 96)])
def test_weight_gradient_of_the_widest_layers(dtype, tokens, n_out, n_in):
    torch = need_gpu()
    print(f"[act8 dw] {dtype} {tokens} tokens, {n_out} x {n_in}", flush=True)
    torch.manual_seed(tokens)
    dt = getattr(torch, dtype)
    x = torch.randint(-8, 9, (tokens, n_in), device="cuda").to(dt)
    dy = torch.randint(-4, 5, (tokens, n_out), device="cuda").to(dt)
    q, s = torch.empty((tokens, n_in), dtype=torch.uint8, device="cuda"), torch.empty((tokens, n_in // 32), dtype=torch.uint8,
                                                                                     device="cuda")
    B.act8_save(x, q, s)
    scratch = torch.empty(max(B.act8_gemm_dw_scratch_bytes(dt, tokens, n_out, n_in), 1), dtype=torch.uint8, device="cuda")
    dw = torch.full((n_out, n_in), float("nan"), device="cuda")
    B.act8_gemm_dw(dy, q, s, dw, scratch)
    torch.cuda.synchronize()
    assert torch.equal(dw, torch.mm(dy.float().t().contiguous(), x.float()))  # integers: exact


@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
@pytest.mark.parametrize("tokens,q,kv,d", [(1, 4096, 4096, 256), (3, 4096, 1, 8), (2, 1, 4096, 64)])
def test_qk_of_the_most_heads(dtype, tokens, q, kv, d):
    G.test_qk_norm_rope(dtype, tokens, q, kv, d, d // 16 * 16, False, True)
