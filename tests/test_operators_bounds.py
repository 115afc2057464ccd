"""Sizes at and beyond what the operators around the blocks take (no GPU): such a call is
refused before anything is enqueued, by the status or the error that names the size."""
import pytest

from paper_2206_04959_amd import binding as B

torch = pytest.importorskip("torch")

BF, U8, F32, I32 = torch.bfloat16, torch.uint8, torch.float32, torch.int32
WRAP = 2 ** 32 + 64  # 64 in 32 bits


def _v(*shape, dtype=BF):
    """A tensor of any shape without memory behind it."""
    return torch.empty(shape, dtype=dtype, device="meta")


def _qk(**change):
    a = dict(qkv=_v(4, 6, 64), gq=_v(64), gk=_v(64), table=_v(9, 32, 2, dtype=F32), out=_v(4, 6, 64), q_heads=2,
             kv_heads=2, seq_len=4, positions=None, **{})
    a.update(change)
    return lambda: B.qk_norm_rope_fwd(a["qkv"], a["gq"], a["gk"], a["table"], a["out"], a["q_heads"], a["kv_heads"],
                                      positions=a["positions"], seq_len=a["seq_len"])


# The entry points' integers have 32 bits (first_id: 64), and ctypes cuts larger ones: a table of
# 2^32 + 64 rows went on as one of 64.
@pytest.mark.parametrize("call", [
    lambda: B.embedding_fwd(_v(4, dtype=I32), _v(WRAP, 64), _v(4, 64)),
    lambda: B.embedding_fwd(_v(1, dtype=I32), _v(9, WRAP), _v(1, WRAP)),
    lambda: B.embedding_fwd(_v(4, dtype=I32), _v(9, 64), _v(4, 64), first_id=2 ** 64 + 3),
    lambda: B.embedding_fwd(_v(4, dtype=I32), _v(9, 64), _v(4, 64), first_id=3 - 2 ** 64),
    lambda: B.embedding_bwd(_v(4, dtype=I32), _v(4, 64), _v(WRAP, 64, dtype=F32)),
    lambda: B.embedding_bwd(_v(1, dtype=I32), _v(1, WRAP), _v(9, WRAP, dtype=F32)),
    lambda: B.embedding_bwd(_v(4, dtype=I32), _v(4, 64), _v(9, 64, dtype=F32), first_id=2 ** 64),
    lambda: B.embedding_scratch_bytes(WRAP, 64),
    lambda: B.embedding_scratch_bytes(4, WRAP),
    lambda: B.embedding_scratch_bytes(4 - 2 ** 32, 64),
    lambda: B.rope_table(_v(WRAP, 32, 2, dtype=F32)),
    lambda: B.rope_table(_v(9, WRAP // 2, 2, dtype=F32)),
    _qk(seq_len=2 ** 32 + 4),
    _qk(seq_len=4 - 2 ** 32),
    _qk(table=_v(WRAP, 32, 2, dtype=F32)),
    _qk(table=_v(9, WRAP // 2, 2, dtype=F32)),
    _qk(qkv=_v(1, WRAP + 4, 64), out=_v(1, WRAP + 4, 64), q_heads=WRAP),
    _qk(qkv=_v(1, 2 * WRAP + 2, 64), out=_v(1, 2 * WRAP + 2, 64), kv_heads=WRAP),
    _qk(qkv=_v(1, 6, WRAP), out=_v(1, 6, WRAP), gq=_v(WRAP), gk=_v(WRAP)),
    lambda: B.qk_norm_rope_scratch_elems(WRAP, 2, 2, 64),
    lambda: B.qk_norm_rope_scratch_elems(4, WRAP, 2, 64),
    lambda: B.act8_save(_v(1, WRAP), _v(1, WRAP, dtype=U8), _v(1, WRAP // 32, dtype=U8)),
    lambda: B.act8_save(_v(WRAP, 64), _v(WRAP, 64, dtype=U8), _v(WRAP, 2, dtype=U8)),
    lambda: B.act8_gemm_dw(_v(4, WRAP), _v(4, 64, dtype=U8), _v(4, 2, dtype=U8), _v(WRAP, 64, dtype=F32)),
    lambda: B.act8_gemm_dw_scratch_bytes(BF, WRAP, 64, 64),
    lambda: B.act8_gemm_dw_scratch_bytes(BF, 4, 64, WRAP),
])
def test_binding_refuses_sizes_that_ctypes_would_cut(call):
    with pytest.raises(ValueError, match="too large"):
        call()


def test_positions_make_seq_len_irrelevant():
    """A sequence length that positions replace is not looked at (the call ends at the device)."""
    with pytest.raises(ValueError, match="one GPU"):
        _qk(positions=_v(4, dtype=I32), seq_len=2 ** 32 + 4)()


P = [0x1000000 * (i + 1) for i in range(12)]  # addresses far apart; nothing reads them
INVALID, SHAPE, ALIGN = -1, -2, -4
LAST = 2 ** 63 - 1  # the largest id


def _embedding(first, rows, y=P[2]):
    L = B.lib()
    return (L.merak_embedding_fwd(0, 1, 10, 64, rows, first, 1.0, P[0], P[1], y, None),
            L.merak_embedding_bwd(0, 1, 10, 64, rows, first, 1.0, P[0], P[1], y, 0, None, None))


def test_the_tables_last_row_has_an_id():
    """Rows whose ids would be beyond 2^63 - 1: id - first_id is formed in 64 bits, so the id
    -2^63 was taken for row 1 of a table that begins at 2^63 - 1."""
    assert (-2 ** 63 - LAST) % 2 ** 64 == 1
    for rows in (2, 100, 2 ** 30):
        assert _embedding(LAST - rows + 2, rows) == (INVALID, INVALID)
        assert _embedding(LAST, rows) == (INVALID, INVALID)
        # the next check is reached by tables that end at the last id
        assert _embedding(LAST - rows + 1, rows, y=P[2] + 4) == (ALIGN, ALIGN)
    assert _embedding(LAST, 1, y=P[2] + 4) == (ALIGN, ALIGN)


# A launch counts its threads in 32 bits, and one of more does only a part of its work, without an
# error.  The least sizes that are too large, each with the largest that is not (whose call ends
# at an unaligned pointer or, here without a GPU, at the launch).
HIP = -6
FAR = [(i + 1) << 44 for i in range(5)]  # addresses that no array of these sizes connects


def _act8(rows, cols):
    L = B.lib()
    return {L.merak_act8_save(0, rows, cols, FAR[0], FAR[1], FAR[2], None),
            L.merak_act8_restore(1, rows, cols, FAR[1], FAR[2], FAR[0], None),
            L.merak_act8_gelu_bwd(0, rows, cols, FAR[0], FAR[1], FAR[2], FAR[3], None, None)}


@pytest.mark.skipif(torch.cuda.is_available(), reason="the allowed sizes would be launched")
@pytest.mark.parametrize("rows,cols,status", [
    (2 ** 30, 32, SHAPE), (2 ** 24, 2 ** 11, SHAPE), (2 ** 30 - 63, 32, SHAPE), (2 ** 30 - 64, 32, HIP),
    (2 ** 24 - 1, 2 ** 11, HIP)])
def test_act8_largest_arrays(rows, cols, status):
    assert _act8(rows, cols) == {status}


@pytest.mark.skipif(torch.cuda.is_available(), reason="the allowed sizes would be launched")
@pytest.mark.parametrize("dtype,tokens,hidden,status", [
    (0, 2 ** 24, 2 ** 13, SHAPE), (0, 2 ** 24 - 1, 2 ** 13, HIP), (1, 2 ** 24, 2 ** 12, SHAPE),
    (1, 2 ** 24 - 1, 2 ** 12, HIP), (0, 2 ** 30, 8, HIP)])
def test_embedding_largest_output(dtype, tokens, hidden, status):
    assert B.lib().merak_embedding_fwd(dtype, 0, tokens, hidden, 10, 0, 1.0, FAR[0], FAR[1], FAR[2], None) == status


@pytest.mark.skipif(torch.cuda.is_available(), reason="the allowed sizes would be launched")
@pytest.mark.parametrize("positions,rope,status", [
    (2 ** 25 - 1, 256, SHAPE), (2 ** 25 - 2, 256, HIP), (2 ** 29, 16, SHAPE), (2 ** 29 - 32, 16, HIP)])
def test_rope_table_largest(positions, rope, status):
    assert B.lib().merak_rope_table(positions, rope, 1e4, FAR[0], None) == status


@pytest.mark.skipif(torch.cuda.is_available(), reason="the allowed sizes would be launched")
@pytest.mark.parametrize("dtype,tokens,n_out,n_in,status", [
    (0, 64, 2 ** 20, 2 ** 20, SHAPE), (1, 64, 2 ** 20, 2 ** 20, SHAPE),  # more output tiles than a launch holds
    (0, 2 ** 25, 2048, 1024, SHAPE),                                     # X is restored first, and too large for it
    (0, 2 ** 25, 512, 1024, HIP), (1, 2 ** 25, 2048, 1024, HIP), (0, 2 ** 24, 2048, 1024, HIP)])
def test_weight_gradient_largest(dtype, tokens, n_out, n_in, status):
    L = B.lib()
    assert L.merak_act8_gemm_dw(dtype, tokens, n_out, n_in, FAR[0], FAR[1], FAR[2], FAR[3], 0, FAR[4], None) == status
