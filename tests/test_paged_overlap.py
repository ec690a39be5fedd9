"""What the paged cache's calls write lies over nothing that they read: refused ahead of every launch, without a GPU."""
import pytest

from paper_2410_16144_amd import binding as B

# addresses that nobody reads: validation comes first
TABLE, POS, START, K, V, Q, KV, OUT, SCRATCH, GQ, GK, ROPE = (n << 32 for n in range(1, 13))
POOL = 10 * 4 * 32 * 64 * 2                                             # bytes
ROWS, OUT_BYTES = 7, 7 * 8 * 64 * 4


def _status(f, *a):
    with pytest.raises(B.BitLinearError) as e:
        f(*a)
    return e.value.status


def _cache(k=K, v=V):
    return B.PagedCache(k, v, 4, 64, 32, 10)


def _rows(table=TABLE, pos=POS, start=START):
    return B.PagedRows(table, pos, start, 5, 3, ROWS, 160)


def _append(k=K, v=V, table=TABLE, pos=POS, start=START, out=OUT, g_q=GQ, g_k=GK, rope=ROPE):
    return _status(B.bl_paged_append, _cache(k, v), _rows(table, pos, start), Q, KV, KV, out, 512, 256, 256, B.BL_F32, B.BL_F32, 8, g_q, g_k, 1e-5, rope)


def _attend(k=K, v=V, table=TABLE, pos=POS, start=START, out=OUT, q=Q, scratch=SCRATCH):
    return _status(B.bl_attn_paged, B.make_attn_paged_args(_cache(k, v), _rows(table, pos, start), q, out, scratch, 8, B.BL_F32))


@pytest.mark.parametrize("written,size", [("k", POOL), ("v", POOL), ("out", OUT_BYTES)])
@pytest.mark.parametrize("read,before", [("table", 3 * 5 * 4), ("pos", 3 * 4), ("start", 4 * 4), ("g_q", 64 * 4), ("g_k", 64 * 4), ("rope", 160 * 32 * 8)])
def test_append(written, size, read, before):
    at = {"k": K, "v": V, "out": OUT}[written]
    step = 8 if read == "rope" else 4
    for off in (0, size - step, step - before):
        assert _append(**{read: at + off}) == B.BL_ERR_SHAPE, off


def test_keys_pages_are_not_values_pages():
    for off in (0, 16, POOL - 16, 16 - POOL):
        assert _append(v=K + off) == B.BL_ERR_SHAPE, off


@pytest.mark.parametrize("read,before", [("table", 3 * 5 * 4), ("pos", 3 * 4), ("start", 4 * 4)])
def test_attention_over_the_description(read, before):
    scratch = B.bl_attn_paged_scratch_bytes(8, 4, 64, 3, ROWS, 160, False)
    for at, size in ((OUT, OUT_BYTES), (SCRATCH, scratch)):
        for off in (0, size - 4, 4 - before):
            assert _attend(**{read: at + off}) == B.BL_ERR_SHAPE, off


def test_scratch_over_queries_and_pages():
    scratch = B.bl_attn_paged_scratch_bytes(8, 4, 64, 3, ROWS, 160, False)
    for name, before in (("q", OUT_BYTES), ("k", POOL), ("v", POOL)):
        for off in (0, scratch - 16, 16 - before):
            assert _attend(**{name: SCRATCH + off}) == B.BL_ERR_SHAPE, (name, off)
