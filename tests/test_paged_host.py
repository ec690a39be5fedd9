"""The paged cache without a GPU: refusals, sizes, structures as the header has them, and what the Python side asks for."""
import ctypes
import os
import subprocess

import pytest
import torch

from paper_2410_16144_amd import binding as B
from paper_2410_16144_amd import decoder

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000   # an aligned address that nobody reads: validation comes first
FAR = 1 << 40


def _st(f, *a):
    with pytest.raises(B.BitLinearError) as e:
        f(*a)
    return e.value.status


def _cache(**kw):
    f = dict(k_pages_dev=P, v_pages_dev=P, n_heads=4, head_dim=64, page_size=32, pages=10)
    return B.PagedCache(**dict(f, **kw))


def _rows(**kw):
    f = dict(table_dev=P, pos_dev=P, start_dev=P, table_width=5, sequences=3, rows=7, max_pos=160)
    return B.PagedRows(**dict(f, **kw))


def test_structures_as_the_header_has_them(tmp_path):
    names = {"bl_paged_cache": B.PagedCache, "bl_paged_rows": B.PagedRows, "bl_paged_append_args": B.PagedAppendArgs, "bl_attn_paged_args": B.AttnPagedArgs}
    lines = "".join('printf("%%zu", sizeof(%s));' % n + "".join('printf(" %%zu", offsetof(%s, %s));' % (n, f[0]) for f in c._fields_) + 'printf("\\n");'
                    for n, c in names.items())
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "bitlinear_decoder.h"\nint main(void) {' + lines +
                   'printf("%d %d %d %d %d %d\\n", BL_PAGE_MIN, BL_PAGE_MAX, BL_PAGED_MAX_HEADS, BL_PAGED_MAX_GROUP, BL_PAGED_MAX_SEQUENCES, BL_PAGED_MAX_POS); return 0;}')
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    said = subprocess.check_output([exe], text=True).splitlines()
    for line, (n, c) in zip(said, names.items()):
        assert [int(x) for x in line.split()] == [ctypes.sizeof(c)] + [getattr(c, f[0]).offset for f in c._fields_], n
    assert [int(x) for x in said[-1].split()] == [B.BL_PAGE_MIN, B.BL_PAGE_MAX, B.BL_PAGED_MAX_HEADS, B.BL_PAGED_MAX_GROUP, B.BL_PAGED_MAX_SEQUENCES, B.BL_PAGED_MAX_POS]


def test_widths():
    want = {4: 32, 32: 32, 36: 48, 48: 48, 52: 64, 64: 64, 68: 96, 96: 96, 100: 128, 128: 128, 132: 192, 192: 192, 196: 256, 256: 256}
    assert {d: B.bl_paged_width(d) for d in want} == want
    for d in (0, -4, 2, 62, 260, 1 << 30):
        assert B.bl_paged_width(d) == 0


def _refusals_of_the_rows(call):
    assert call(_cache(k_pages_dev=None)) == call(_cache(v_pages_dev=None)) == call(rows=_rows(table_dev=None)) == call(rows=_rows(pos_dev=None)) == B.BL_ERR_NULL
    for kw in (dict(n_heads=0), dict(n_heads=3), dict(n_heads=1025), dict(head_dim=62), dict(head_dim=0), dict(head_dim=260), dict(page_size=8), dict(page_size=48),
               dict(page_size=8192), dict(page_size=0), dict(page_size=-32), dict(pages=0), dict(pages=-1)):
        assert call(_cache(**kw)) == B.BL_ERR_SHAPE, kw
    for kw in (dict(sequences=0), dict(sequences=1025), dict(rows=0), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(table_width=0), dict(max_pos=0), dict(max_pos=161),
               dict(start_dev=None), dict(max_pos=2147483647), dict(table_width=-1)):
        assert call(rows=_rows(**kw)) == B.BL_ERR_SHAPE, kw
    for c in (_cache(k_pages_dev=P + 8), _cache(v_pages_dev=P + 2)):
        assert call(c) == B.BL_ERR_ALIGN
    for kw in (dict(table_dev=P + 2), dict(pos_dev=P + 1), dict(start_dev=P + 2)):
        assert call(rows=_rows(**kw)) == B.BL_ERR_ALIGN


def test_refusals_of_append():
    def call(cache=None, rows=None, **kw):
        a = dict(q=P, k=P, v=P, q_out=FAR, ld_q=512, ld_k=256, ld_v=256, dt=B.BL_F32, q_dt=B.BL_F32, n_q=8, g_q=P, g_k=P, eps=1e-5, table=P)
        a.update(kw)
        return _st(B.bl_paged_append, cache or _cache(), rows or _rows(), *a.values())
    _refusals_of_the_rows(call)
    for name in ("q", "k", "v", "q_out"):
        assert call(**{name: 0}) == B.BL_ERR_NULL
    assert _st(B.bl_paged_append, None, _rows(), P, P, P, FAR, 512, 256, 256, 0, 0, 8) == _st(B.bl_paged_append, _cache(), None, P, P, P, FAR, 512, 256, 256, 0, 0, 8) == B.BL_ERR_NULL
    for kw in (dict(n_q=0), dict(n_q=6), dict(n_q=-4), dict(n_q=4 * 65), dict(ld_q=511), dict(ld_k=255), dict(ld_v=0), dict(ld_q=1 << 62), dict(n_q=12)):
        assert call(**kw) == B.BL_ERR_SHAPE, kw
    for kw in (dict(dt=2), dict(q_dt=-1)):
        assert call(**kw) == B.BL_ERR_DTYPE
    for kw in (dict(q=P + 2), dict(k=P + 1, dt=B.BL_BF16), dict(v=P + 2), dict(q_out=FAR + 8), dict(g_q=P + 2), dict(g_k=P + 2), dict(table=P + 4)):
        assert call(**kw) == B.BL_ERR_ALIGN, kw
    # queries go to memory of their own
    out_bytes = 7 * 512 * 4
    for off in (0, 16, -16, out_bytes - 16, 16 - out_bytes):
        assert call(q=FAR + off) == B.BL_ERR_SHAPE, off
    assert call(k=FAR + 64) == call(v=FAR) == B.BL_ERR_SHAPE
    assert call(q=FAR - out_bytes, g_q=P + 2) == call(q=FAR + out_bytes, g_q=P + 2) == B.BL_ERR_ALIGN      # (nothing wrong with q)
    assert call(_cache(k_pages_dev=FAR + 16)) == call(_cache(v_pages_dev=FAR - 16)) == B.BL_ERR_SHAPE
    assert call(_cache(n_heads=1), _rows(rows=1 << 24), n_q=64, ld_q=4096) == B.BL_ERR_SHAPE               # 2^32 threads


def test_refusals_of_the_attention():
    def call(cache=None, rows=None, n_q=8, dt=B.BL_F32, **kw):
        a = dict(q=P, out=FAR, scratch=P)
        a.update(kw)
        return _st(B.bl_attn_paged, B.make_attn_paged_args(cache or _cache(), rows or _rows(), *a.values(), n_q, dt))
    _refusals_of_the_rows(call)
    for name in ("q", "out", "scratch"):
        assert call(**{name: 0}) == B.BL_ERR_NULL
    assert _st(B.bl_attn_paged, B.make_attn_paged_args(None, _rows(), P, FAR, P, 8, 0)) == _st(B.bl_attn_paged, B.make_attn_paged_args(_cache(), None, P, FAR, P, 8, 0)) == B.BL_ERR_NULL
    for n_q in (0, 6, -4, 4 * 65):
        assert call(n_q=n_q) == B.BL_ERR_SHAPE
    assert call(dt=2) == B.BL_ERR_DTYPE
    for kw in (dict(q=P + 4), dict(out=FAR + 4), dict(scratch=P + 64)):
        assert call(**kw) == B.BL_ERR_ALIGN, kw
    for off in (0, 8, 7 * 512 * 4 - 8, 8 - 7 * 512 * 4):
        assert call(q=FAR + off) == B.BL_ERR_SHAPE
    pool = 10 * 4 * 32 * 64 * 2
    for far in (dict(k_pages_dev=FAR + 16), dict(v_pages_dev=FAR - pool + 16)):
        assert call(_cache(**far)) == B.BL_ERR_SHAPE, far
    assert call(_cache(k_pages_dev=FAR - pool), q=P + 4) == B.BL_ERR_ALIGN                                 # (nothing wrong with the pages)
    assert call(scratch=FAR + 256) == call(scratch=FAR - 256) == B.BL_ERR_SHAPE
    assert call(_cache(n_heads=1), _rows(rows=1 << 24), n_q=64) == B.BL_ERR_SHAPE                          # 2^32 threads


def test_scratch():
    f = B.bl_attn_paged_scratch_bytes
    for bad in ((6, 4, 64, 3, 7, 160, 0), (8, 0, 64, 3, 7, 160, 0), (8, 4, 62, 3, 7, 160, 0), (8, 4, 64, 0, 7, 160, 0), (8, 4, 64, 1025, 7, 160, 0), (8, 4, 64, 3, 0, 160, 0),
                (8, 4, 64, 3, 7, 0, 0), (8, 4, 64, 3, 7, 160, 1), (4 * 65, 4, 64, 3, 7, 160, 0)):
        assert f(*bad) == 0, bad
    # the counters of any call, whatever else
    for args in ((8, 4, 64, 3, 7, 160, 0), (8, 4, 64, 3, 3, 160, 1), (8, 4, 64, 1024, 1024, 1 << 20, 1), (8, 4, 256, 1, 4096, 1 << 20, 0)):
        assert f(*args) >= 1 << 16 and f(*args) % 16 == 0
    # no figures where no walk can be shared
    assert f(8, 4, 64, 3, 3, 160, 1) == 1 << 16
    # and memory in bounds at the largest
    assert f(64, 1, 256, 1024, 1024, 1 << 30, 1) < 1 << 33 and f(64, 1, 256, 1, 1 << 20, 1 << 30, 0) < 1 << 33
    assert f(8, 4, 64, 3, 7, (1 << 30) + 1, 0) == 0


def test_what_the_python_side_asks_for():
    for kw in (dict(page_size=24), dict(page_size=8), dict(head_dim=6), dict(pages=0), dict(n_heads=0)):
        a = dict(n_heads=2, head_dim=64, page_size=16, pages=4)
        a.update(kw)
        with pytest.raises(B.BitLinearError) as e:
            decoder.PagedCache(**a, device="cpu")
        assert e.value.status == B.BL_ERR_SHAPE
    c = decoder.PagedCache(2, 100, 16, 4, "cpu")
    assert c.k.shape == c.v.shape == (4, 2, 16, 128) and c.k.dtype == torch.bfloat16
    with pytest.raises(AssertionError):
        decoder.PagedCache(2, 100, 16, 4, "cpu", k=c.k[:, :, :, :100], v=c.v)
    table, pos = torch.zeros((3, 2), dtype=torch.int32), torch.zeros(3, dtype=torch.int32)
    r = decoder.PagedRows(table, pos, 32)
    assert r.rows == r.sequences == 3 and r.args.start_dev is None and r.args.table_width == 2
    with pytest.raises(ValueError):
        decoder.PagedRows(table, pos, 32, start=torch.zeros(4, dtype=torch.int32))
    for bad in (dict(table=table.long()), dict(pos=pos[:2]), dict(start=torch.zeros(3, dtype=torch.int32), rows=3), dict(table=table.t())):
        a = dict(table=table, pos=pos, max_pos=32)
        a.update(bad)
        with pytest.raises(AssertionError):
            decoder.PagedRows(**a)
    for bad in (dict(max_pos=0), dict(max_pos=(1 << 32) + 5), dict(rows=(1 << 32) + 3, start=torch.zeros(4, dtype=torch.int32)), dict(pos=pos[:0], table=table[:0])):
        with pytest.raises(B.BitLinearError) as e:
            decoder.PagedRows(**dict(dict(table=table, pos=pos, max_pos=32), **bad))
        assert e.value.status == B.BL_ERR_SHAPE
    q = torch.zeros((3, 400))
    with pytest.raises(AssertionError):
        decoder.attn_paged(q, c, r, torch.zeros(1 << 20, dtype=torch.uint8))       # not on a device
    with pytest.raises(AssertionError):
        c.append(q, q[:, :200], q[:, :200], r, None)
