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
