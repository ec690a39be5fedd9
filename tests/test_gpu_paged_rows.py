"""Whose rows a call of the paged cache has, where starts fall or say nothing of use: what one sound sequence alone claims is right, everything else as it was."""
import pytest

from test_gpu_paged import F, G, H, U, Server, _append_want, _close, _gen, _queries, _want, dec, dev   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _owners(start, pos, rows, max_pos):
    """Each row's sequence; None where none claims it, ... where several do."""
    of = [None] * rows
    for b in range(len(pos)):
        first, end = start[b], start[b + 1]
        if first >= 0 and first <= end <= rows and pos[b] >= 0 and pos[b] + end - first <= max_pos:
            for t in range(first, end):
                of[t] = b if of[t] is None else ...
    return of


FEW = [[0, 3, -1, 5, 8], [0, 3, 9, 9, 8], [4, 2, 2, 8, 8], [0, 0, 0, 0, 0], [8, 8, 8, 8, 8], [0, 2147483647, -2147483648, 5, 8], [0, 9, 3, 5, 8], [5, 7, 0, 2, 4], [-1, 2, 6, 4, 8]]


def _many(sequences, seed):
    """Starts of more sequences than lanes, rising by 0 to 2, but for some that fall, or say what is not there."""
    g = _gen(seed)
    start = [0] + torch.randint(0, 3, (sequences,), generator=g).cumsum(0).tolist()
    for i in torch.randint(1, sequences, (5,), generator=g).tolist():
        start[i] = [-7, 1 << 30, 0, start[-1] + 1, -1][i % 5]
    return start


@pytest.mark.parametrize("start", FEW + [_many(70, 1), _many(130, 2), _many(700, 4), _many(1024, 4)], ids=lambda s: "%d" % len(s) if len(s) > 9 else "-".join(map(str, s)))
@pytest.mark.parametrize("what", ["append", "attention"])
def test_starts_that_fall_hide_nobody_elses_rows(dev, dec, start, what):
    heads, n, d, page, max_pos = 4, 2, 32, 16, 32
    B = len(start) - 1
    rows = max(8, start[-1])
    g = _gen(len(start))
    pos = torch.randint(0, 14, (B,), generator=g).tolist()
    pos[B // 2] = max_pos                                               # (one that takes no part for its position)
    srv = Server(dec, dev, n, d, page, [max_pos] * B, 5, unowned=0.25)
    of = _owners(start, pos, rows, max_pos)
    claimed = sum(e - s for s, e, p in zip(start, start[1:], pos) if 0 <= s <= e <= rows and 0 <= p <= max_pos - (e - s))
    assert claimed <= rows
    calls = dec.PagedRows(srv.lines.to(dev)[:, :2].contiguous(), torch.tensor(pos, dtype=torch.int32, device=dev), max_pos,
                          start=torch.tensor(start, dtype=torch.int32, device=dev), rows=rows)
    out = torch.full((rows, heads * d), -7.0, device=dev)
    if what == "append":
        x = torch.randn((rows, (heads + 2 * n) * d), generator=g).to(dev)
        k0, v0 = srv.cache.k.clone(), srv.cache.v.clone()
        srv.cache.append(x[:, :heads * d], x[:, heads * d:(heads + n) * d], x[:, (heads + n) * d:], calls, None, q_out=out)
        want = torch.full_like(out, -7.0)
        for t, b in enumerate(of):
            if b is ...:
                continue
            if b is not None:
                want[t] = x[t, :heads * d]
                p = pos[b] + t - start[b]
                where = int(srv.lines[b, p // page])
                k0[where, :, p % page, :d] = x[t, heads * d:(heads + n) * d].to(G).view(n, d)
                v0[where, :, p % page, :d] = x[t, (heads + n) * d:].to(G).view(n, d)
        alone = torch.tensor([b is not ... for b in of], device=dev)
        assert bool((out[alone] == want[alone]).all())
        if alone.all():
            assert torch.equal(srv.cache.k, k0) and torch.equal(srv.cache.v, v0)
        return
    for b in range(B):
        srv.fill(b, max_pos)
    q = _queries(g, rows, heads, d, F, dev)
    dec.attn_paged(q, srv.cache, calls, dec.paged_scratch(heads, srv.cache, calls), out=out)
    for b in range(B):
        mine = [t for t in range(rows) if of[t] == b]
        if mine:
            seen = torch.tensor([pos[b] + 1 + t - start[b] for t in mine])
            want, S, V = _want(q[mine].double().cpu().view(len(mine), heads, d), srv.k[b], srv.v[b], heads // n, seen)
            _close(out[mine], want, S, V, d, F)
    nobody = torch.tensor([b is None for b in of], device=dev)
    assert bool((out[nobody] == -7.0).all())


@pytest.mark.parametrize("single", [True, False])
def test_buffers_that_lie_side_by_side(dev, dec, single):
    """Nothing overlaps where one ends as the next begins."""
    heads, n, d, page, T = 4, 2, 64, 16, 3
    counts = dict(k=12 * n * page * d * 2, v=12 * n * page * d * 2, scratch=0, q=T * heads * d * 4, out=T * heads * d * 4, q1=T * heads * d * 4, table=3 * 4 * 4, pos=16, start=16,
                  g=d * 4, rope=64 * d * 4)
    counts["scratch"] = dec.B.bl_attn_paged_scratch_bytes(heads, n, d, 3, T, 64, single)
    memory, views, at = torch.zeros(sum(counts.values()), dtype=torch.uint8, device=dev), {}, 0
    for name, size in counts.items():
        views[name] = memory[at:at + size]
        at += size
    k, v = (views[x].view(G).view(12, n, page, d) for x in "kv")
    cache = dec.PagedCache(n, d, page, 12, dev, k=k, v=v)
    q, out, q1 = (views[x].view(F).view(T, heads * d) for x in ("q", "out", "q1"))
    table, pos, start = views["table"].view(torch.int32).view(3, 4), views["pos"].view(torch.int32)[:3], views["start"].view(torch.int32)
    table.copy_(torch.arange(12).view(3, 4))                             # (pages that sequences share are nobody's to write)
    start.copy_(torch.arange(4))
    g, rope = views["g"].view(F), views["rope"].view(F).view(64, d // 2, 2)
    g.fill_(1.0)
    rope.copy_(dec.rope_table(d, 64, dev))
    rows = dec.PagedRows(table, pos, 64, start=None if single else start, rows=T)
    q.copy_(torch.randn(q.shape, generator=_gen(1)))
    x = torch.randn((T, n * d), generator=_gen(2)).to(dev)
    cache.append(q, x, x, rows, rope, g_q=g, g_k=g, q_out=q1)
    dec.attn_paged(q1, cache, rows, views["scratch"], out=out)
    # Each sees itself alone: its weight, whatever it is, is divided out.  Three pieces' products added up, the sum's reciprocal and a product with it: five roundings.
    want = x.to(G).float().view(T, n, 1, d).expand(-1, -1, heads // n, -1).reshape(T, -1)
    wrong = int(((out - want).abs() > 6 * U * want.abs()).sum())
    assert wrong == 0
