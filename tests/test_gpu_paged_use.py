"""The paged cache as a server uses it: projections, append and attention one after the other, in captured graphs, on other streams, in every form of
the attention, at the limits, and what is refused.  Tolerances and the plain formulas: test_gpu_paged.py."""
import math

import numpy as np
import pytest

from test_gpu_paged import F, G, H, U, Server, _append_want, _attend, _close, _gen, _queries, _want, dec, dev   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _int(dev, *x):
    return torch.tensor(x, dtype=torch.int32, device=dev)


def _held(cache, line, count, d):
    """Keys and values of a sequence's first `count` positions as the pools have them, in 64 bits."""
    at = torch.arange(count)
    page, slot = line[at // cache.page_size].long().to(cache.k.device), (at % cache.page_size).to(cache.k.device)
    return tuple(pool[page, :, slot, :d].double().cpu() for pool in (cache.k, cache.v))


class Layer:
    """Projections with ternary weights around the cache: x [rows, K] -> [rows, K]."""

    def __init__(self, dec, dev, heads, n, d, seed):
        from paper_2410_16144_amd import ops
        g = _gen(seed)
        self.dec, self.ops, self.heads, self.n, self.d, self.K = dec, ops, heads, n, d, heads * d
        pack = lambda N, K: ops.pack_ternary(torch.randint(-1, 2, (N, K), generator=g).to(torch.int8).to(dev), 1.3 / math.sqrt(K))
        self.wq, self.wk, self.wv, self.wo = pack(heads * d, self.K), pack(n * d, self.K), pack(n * d, self.K), pack(self.K, heads * d)
        self.g_q, self.g_k = ((torch.rand(d, generator=g) + 0.5).to(dev) for _ in range(2))

    def projections(self, x):
        return self.ops.gemm_batch([self.wq, self.wk, self.wv], self.ops.quant_act(x))

    def __call__(self, x, cache, rows, table, scratch, q_dtype=F):
        q, k, v = self.projections(x)
        q = cache.append(q, k, v, rows, table, g_q=self.g_q, g_k=self.g_k, q_dtype=q_dtype)
        out = self.dec.attn_paged(q, cache, rows, scratch)
        return self.ops.gemm(self.wo, self.ops.quant_act(out))


@pytest.mark.parametrize("q_dtype", [F, G])
def test_a_server_with_requests_that_come_and_go(dev, dec, q_dtype):
    """Prompts, mixtures of pieces and single tokens, then single tokens alone, over one pool; every step against the formulas."""
    heads, n, d, page = 8, 2, 64, 16
    layer, g = Layer(dec, dev, heads, n, d, 40), _gen(41)
    cache = dec.PagedCache(n, d, page, 64, dev)
    table = dec.rope_table(d, 256, dev)
    lines = torch.randperm(64, generator=g)[:4 * 16].view(4, 16).to(torch.int32)
    scratch = dec.paged_scratch(heads, cache, dec.PagedRows(lines.to(dev), _int(dev, 0, 0, 0, 0), 256, start=_int(dev, 0, 0, 0, 0, 0), rows=300))
    done, keys, values = [0] * 4, [[] for _ in range(4)], [[] for _ in range(4)]
    for new in ((50, 0, 7, 0), (1, 33, 1, 0), (1, 1, 90, 3), (5, 1, 1, 130), None, None, None):
        single, new = new is None, new or (1, 1, 1, 1)
        T = sum(new)
        x = torch.randn((T, layer.K), generator=g).to(dev)
        start = None if single else torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=dev)
        rows = dec.PagedRows(lines.to(dev), _int(dev, *done), 256, start=start, rows=T)
        q, k, v = layer.projections(x)
        q1 = cache.append(q, k, v, rows, table, g_q=layer.g_q, g_k=layer.g_k, q_dtype=q_dtype)
        out = dec.attn_paged(q1, cache, rows, scratch)
        y = layer.ops.gemm(layer.wo, layer.ops.quant_act(out))
        assert y.shape == x.shape and torch.isfinite(y).all()
        t = 0
        for b, m in enumerate(new):
            if not m:
                continue
            angles = table[done[b]:done[b] + m].double().cpu()
            want_q, size = _append_want(q[t:t + m].double().cpu(), heads, d, layer.g_q.double().cpu(), dec.EPS, angles)
            have_q = q1[t:t + m].double().cpu().view(m, heads, d)
            assert ((have_q - want_q).abs() <= 30 * U * size + (H if q_dtype == G else 0) * (want_q.abs() + 30 * U * size)).all()
            done[b] += m
            have_k, have_v = _held(cache, lines[b], done[b], d)
            want_k, size = _append_want(k[t:t + m].double().cpu(), n, d, layer.g_k.double().cpu(), dec.EPS, angles)
            assert ((have_k[-m:] - want_k).abs() <= 30 * U * size + H * (want_k.abs() + 30 * U * size)).all()
            assert torch.equal(have_v[-m:], v[t:t + m].to(G).double().cpu().view(m, n, d))
            keys[b].append(have_k[-m:])
            values[b].append(have_v[-m:])
            assert torch.equal(have_k, torch.cat(keys[b])) and torch.equal(have_v, torch.cat(values[b]))   # (nobody wrote what was there)
            want, S, V = _want(have_q, have_k, have_v, heads // n, done[b] - m + 1 + torch.arange(m))
            _close(out[t:t + m], want, S, V, d, q_dtype)
            t += m


# ---------------------------------------------------------------------------------------------------- graphs and streams

def test_a_captured_step_serves_other_lengths_pages_and_rows(dev, dec):
    """One graph of two layers' steps; between its replays the inputs, positions, starts and the table change, and eager work runs."""
    heads, n, d, page, T = 8, 2, 64, 16, 48
    layers = [Layer(dec, dev, heads, n, d, 50 + i) for i in range(2)]
    g = _gen(52)
    table = dec.rope_table(d, 512, dev)
    lines, pos, start = torch.zeros((3, 32), dtype=torch.int32, device=dev), _int(dev, 0, 0, 0), _int(dev, 0, 1, 2, 3)
    caches = [[dec.PagedCache(n, d, page, 96, dev) for _ in layers] for _ in range(2)]       # the graph's and the eager calls'
    rows = dec.PagedRows(lines, pos, 512, start=start, rows=T)
    scratch = [dec.paged_scratch(heads, caches[0][0], rows) for _ in range(2)]
    x, y = torch.zeros((T, heads * d), device=dev), torch.zeros((T, heads * d), device=dev)

    def step(cache, own):
        z = x
        for layer, c in zip(layers, cache):
            q, k, v = layer.projections(z)
            q = c.append(q, k, v, rows, table, g_q=layer.g_q, g_k=layer.g_k)
            out = torch.zeros_like(q)                                                        # (rows of nobody stay zero)
            dec.attn_paged(q, c, rows, own, out=out)
            z = layer.ops.gemm(layer.wo, layer.ops.quant_act(out))
        return z
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[0], scratch[0])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y.copy_(step(caches[0], scratch[0]))
    done = [0, 0, 0]
    for i, new in enumerate(((40, 1, 7), (1, 0, 47), (0, 0, 1), (16, 16, 16), (1, 1, 1), (3, 40, 5), (1, 1, 1))):
        if i in (0, 3):                                                                      # other pages from here on
            lines.copy_(torch.randperm(96, generator=g).to(torch.int32).view(3, 32))
            done = [0, 0, 0]
        pos.copy_(_int(dev, *done))
        start.copy_(torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32))
        x.copy_(torch.randn(x.shape, generator=g))
        want = step(caches[1], scratch[1])
        graph.replay()
        assert torch.equal(y, want), i
        for a, b in zip(*caches):
            assert torch.equal(a.k.view(torch.int16), b.k.view(torch.int16)) and torch.equal(a.v.view(torch.int16), b.v.view(torch.int16))
        done = [a + b for a, b in zip(done, new)]
        torch.cuda.synchronize()


def test_a_token_loop_that_advances_its_own_positions(dev, dec):
    heads, n, d = 4, 2, 128
    srv = Server(dec, dev, n, d, 32, [200, 60, 400], 60)
    for b, m in enumerate((100, 3, 333)):
        srv.fill(b, m)
    pos = _int(dev, 100, 3, 333)
    rows = dec.PagedRows(srv.lines.to(dev), pos, srv.max_pos)
    x, out = torch.zeros((3, (heads + 2 * n) * d), device=dev), torch.zeros((3, heads * d), device=dev)

    def token():
        dec.attn_paged(srv.cache.append(x[:, :heads * d], x[:, heads * d:-n * d], x[:, -n * d:], rows, None, q_out=q), srv.cache, rows, scratch, out=out)
    q = torch.zeros((3, heads * d), device=dev)
    scratch = dec.paged_scratch(heads, srv.cache, rows)
    call = dec.AttentionPaged(heads, srv.cache, rows, q, scratch=scratch)
    graph = torch.cuda.CUDAGraph()
    token()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        token()
        call.launch()                                                    # (the same again, prepared)
        pos.add_(1)
    for i in range(6):
        x.copy_(torch.randn(x.shape, generator=srv.g))
        graph.replay()
        for b in range(3):
            srv.k[b] = torch.cat([srv.k[b], x[b, heads * d:-n * d].to(G).double().cpu().view(1, n, d)])
            srv.v[b] = torch.cat([srv.v[b], x[b, -n * d:].to(G).double().cpu().view(1, n, d)])
            want, S, V = _want(x[b, :heads * d].double().cpu().view(1, heads, d), srv.k[b], srv.v[b], 2, torch.tensor([srv.k[b].shape[0]]))
            _close(out[b], want, S, V, d, F)
        assert torch.equal(call.out, out)
    assert pos.tolist() == [106, 9, 339]


@pytest.mark.parametrize("dtype", [F, G])
def test_two_streams_with_a_scratch_each(dev, dec, dtype):
    """Shared walks of two streams at once, and two captured graphs replayed at once."""
    heads, n, d = 8, 2, 128
    srv = Server(dec, dev, n, d, 64, [6000, 3000], 70)
    for b, m in enumerate((6000, 3000)):
        srv.fill(b, m)
    calls = []
    for before, new, single in (([5999, 2000], [1, 1], True), ([5000, 100], [9, 60], False)):
        rows = srv.rows(dec, before, new, single)
        q = _queries(srv.g, sum(new), heads, d, dtype, dev)
        calls.append((q, rows, dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows))))
    streams = [torch.cuda.Stream() for _ in calls]
    scratch = [dec.paged_scratch(heads, srv.cache, c[1]) for c in calls]
    torch.cuda.synchronize()
    outs = [[], []]
    for _ in range(10):
        for i, (q, rows, _) in enumerate(calls):
            with torch.cuda.stream(streams[i]):
                outs[i].append(dec.attn_paged(q, srv.cache, rows, scratch[i]))
    torch.cuda.synchronize()
    assert all(torch.equal(o, calls[i][2]) for i in range(2) for o in outs[i])
    graphs, held = [], []
    for i, (q, rows, _) in enumerate(calls):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i]):
            held.append(dec.attn_paged(q, srv.cache, rows, scratch[i]))
    for _ in range(5):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                held[i].zero_()
                graphs[i].replay()
        torch.cuda.synchronize()
        assert all(torch.equal(held[i], calls[i][2]) for i in range(2))
    assert not any(s[:1 << 16].any() for s in scratch)


def test_prepared_eager_and_bound_calls_give_the_same_bits(dev, dec, monkeypatch):
    """AttentionPaged, the native calls and the ctypes binding behind them."""
    heads, n, d = 6, 3, 96
    srv = Server(dec, dev, n, d, 16, [300, 70], 80)
    for b, m in enumerate((290, 60)):
        srv.fill(b, m)
    x = torch.randn((12, (heads + 2 * n) * d), generator=srv.g).to(dev)
    table = dec.rope_table(d, srv.max_pos, dev)
    for dtype in (F, G):
        for before, new, single in (([280, 50], [1, 1], True), ([280, 50], [9, 3], False)):
            rows = srv.rows(dec, before, new, single)
            y = x[:sum(new)].to(dtype)
            args = (y[:, :heads * d], y[:, heads * d:(heads + n) * d], y[:, (heads + n) * d:], rows, table)
            scratch = dec.paged_scratch(heads, srv.cache, rows)
            got = []
            for bound in (False, True):
                with monkeypatch.context() as m:
                    if bound:
                        m.setattr(dec.B, "calls", lambda: False)
                    q = srv.cache.append(*args)
                    out = dec.attn_paged(q, srv.cache, rows, scratch)
                    call = dec.AttentionPaged(heads, srv.cache, rows, q, scratch=scratch)
                    assert torch.equal(call.launch(), out)
                    got.append((q, out, srv.cache.k.clone()))
            assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
            assert torch.equal(got[0][2].view(torch.int16), got[1][2].view(torch.int16))


# ---------------------------------------------------------------------------------------------------- every form of the attention

# (rows that the call has room for and nobody has make the host expect so many tiles: by one and by two of 64 rows on a compute unit, 128 rows)
@pytest.mark.parametrize("extra", [0, 2200, 7000])
@pytest.mark.parametrize("heads,n,d", [(8, 2, 128), (8, 2, 96), (8, 2, 64), (8, 2, 120), (8, 2, 36), (8, 2, 32), (8, 2, 192), (8, 2, 256)])
@pytest.mark.parametrize("page,before,new", [(16, [0, 100, 0, 3], [130, 1, 0, 64]), (64, [3000, 17], [40, 35])])
def test_packed_sequences_in_every_form(dev, dec, heads, n, d, page, before, new, extra):
    _attend(dec, dev, heads, n, d, page, before, new, G, 90 + d, extra=extra)


def _with_odd_values(dec, dev, d, before, new, at, dtype, extra=0, single=False):
    """Values of the positions `at` that are not finite; a row is what the formula makes of those that it sees."""
    heads, n = 8, 2
    srv = Server(dec, dev, n, d, 16, [before + new], 95)
    srv.fill(0, before + new)
    clean = srv.v[0].clone()
    odd = torch.zeros((before + new, n, d))
    for i, p in enumerate(at):
        for e, x in ((i, math.inf), (d - 1 - i, -math.inf), (d // 2 + i, math.nan), (20, math.inf if i % 2 else -math.inf)):
            odd[p, :, e] = x
            clean[p, :, e] = 0
        srv.cache.v[int(srv.lines[0, p // 16]), :, p % 16, :d] = (clean[p] + odd[p].double()).to(G).to(dev)
    q = torch.zeros((new + extra, heads * d), dtype=dtype, device=dev)
    q[:new] = _queries(srv.g, new, heads, d, dtype, dev)
    rows = srv.rows(dec, [before], [new], single, total=new + extra)
    out = dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows))[:new].double().cpu().view(new, heads, d)
    seen = before + 1 + torch.arange(new)
    want, S, V = _want(q[:new].double().cpu().view(new, heads, d), srv.k[0], clean, heads // n, seen)
    touched = torch.zeros((new, n, d))
    for p in at:
        row = torch.where(seen > p, 1.0, 0.0)[:, None, None]
        touched = touched + torch.where(row.bool(), odd[p][None], torch.zeros(()))           # (inf - inf and NaN are NaN)
    touched = touched.repeat_interleave(heads // n, 1)
    finite = torch.isfinite(touched)
    assert torch.equal(out.isnan(), touched.isnan())
    assert torch.equal(out[touched.isinf()].float(), touched[touched.isinf()])
    _close(torch.where(finite, out, want), want, S, V, d, dtype)


@pytest.mark.parametrize("extra", [0, 2200, 7000])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("before,new", [(0, 65), (100, 40), (63, 1), (500, 130)])
def test_values_that_are_not_finite_in_every_form(dev, dec, d, before, new, extra):
    at = sorted({before + new - 1, before + new // 2, before + new // 3, max(0, before - 1)})
    _with_odd_values(dec, dev, d, before, new, at, G, extra)


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("d", [48, 64, 100, 128, 256])
@pytest.mark.parametrize("before,new,at", [(900, 1, [5, 300, 700]), (900, 1, [899]), (900, 70, [0, 899]), (2600, 5, [64, 1300, 2500]), (90, 90, [100, 170])])
@pytest.mark.parametrize("single", [True, False])
def test_values_that_are_not_finite_far_behind(dev, dec, dtype, d, before, new, at, single):
    """Where every row sees the whole chunk: the pieces of a weight must not make NaN of an infinity."""
    if single and new > 1:
        before, new = before + new - 1, 1
    _with_odd_values(dec, dev, d, before, new, at, dtype, single=single)


# ---------------------------------------------------------------------------------------------------- limits

@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("heads,n,d,page,before,new", [
    (4, 1, 64, 256, [70000], None), (1, 1, 128, 4096, [40000, 1], None), (4, 1, 64, 256, [60000], [5]), (40, 1, 32, 4096, [30000], None), (1, 1, 128, 64, [9000], [64]),
    (1024, 1024, 4, 16, [40, 0, 17], None), (1024, 1024, 4, 16, [40, 0], [5, 20]), (2, 1, 32, 16, [i % 40 for i in range(1024)], None),
    (2, 1, 32, 16, [i % 40 for i in range(1024)], [i % 3 for i in range(1024)])])
def test_the_largest_walks_heads_and_sequences(dev, dec, dtype, heads, n, d, page, before, new):
    _attend(dec, dev, heads, n, d, page, before, new or [1] * len(before), dtype, 100 + d, single=new is None)


def test_positions_up_to_the_last(dev, dec):
    """The table's last entry for position 2^30 - 1, and a walk over millions of positions whose pages are few: its weights are those of one page each."""
    n, d, page, width = 1, 8, 4096, 1 << 18
    cache = dec.PagedCache(n, d, page, 4, dev)
    g = _gen(110)
    cache.k[..., :d] = torch.randn((4, n, page, d), generator=g).to(G).to(dev)
    cache.v[..., :d] = torch.randn((4, n, page, d), generator=g).to(G).to(dev)
    table = torch.zeros((1, width), dtype=torch.int32)
    table[0, ::3], table[0, -1] = 1, 3
    x = torch.randn((1, 3 * d), generator=g).to(dev)
    rows = dec.PagedRows(table.to(dev), _int(dev, (1 << 30) - 1), 1 << 30)
    k0, v0 = cache.k.clone(), cache.v.clone()
    cache.append(x[:, :d], x[:, d:2 * d], x[:, 2 * d:], rows, None)
    k0[3, 0, page - 1, :d], v0[3, 0, page - 1, :d] = x[0, d:2 * d].to(G), x[0, 2 * d:].to(G)
    assert torch.equal(cache.k, k0) and torch.equal(cache.v, v0)
    pages = 1500                                                                             # 6.1 million positions
    rows = dec.PagedRows(table.to(dev), _int(dev, pages * page - 1), 1 << 30)
    q = torch.randn((1, 2 * d), generator=g).to(dev)
    out = dec.attn_paged(q, cache, rows, dec.paged_scratch(2, cache, rows))
    count = torch.bincount(table[0, :pages].long(), minlength=4).double()
    k, v = (t[:, 0, :, :d].double().cpu().reshape(4 * page, d) for t in (cache.k, cache.v))
    for h in range(2):
        s = k @ q[0, h * d:(h + 1) * d].double().cpu() / math.sqrt(d)
        w = torch.exp(s - s.max()) * count.repeat_interleave(page)
        want = (w @ v) / w.sum()
        # a lane adds up 6.1e6 / (256 parts * 4 waves * 4 lanes) weights of which each sum is rounded, relative to what is summed up; outputs: four times as many
        bound = 4 * (pages * page / 1024 + 300) * U * (w @ v.abs()) / w.sum() + 100 * U
        assert ((out[0, h * d:(h + 1) * d].double().cpu() - want).abs() <= bound).all()


@pytest.mark.parametrize("start", [[0, 8, 0, 8, 8], [0, 8, 0, 3, 8], [0, 8, 8, 0, 8]])
def test_starts_that_overlap_stay_inside(dev, dec, start):
    """Rows that two sequences claim are one's or the other's; all else is as it was, the scratch is as usable as before."""
    heads, n, d = 4, 2, 64
    srv = Server(dec, dev, n, d, 16, [3000] * 4, 120)
    for b in range(4):
        srv.fill(b, 3000)
    q = _queries(srv.g, 8, heads, d, F, dev)
    rows = dec.PagedRows(srv.lines.to(dev), _int(dev, 2000, 9, 1000, 20), srv.max_pos, start=_int(dev, *start), rows=8)
    guard = torch.full((24, heads * d), -7.0, device=dev)
    scratch = dec.paged_scratch(heads, srv.cache, rows)
    dec.attn_paged(q, srv.cache, rows, scratch, out=guard[8:16])
    assert (guard[:8] == -7).all() and (guard[16:] == -7).all()
    assert not scratch[:1 << 16].any()
    good = srv.rows(dec, [2990, 0, 0, 0], [8, 0, 0, 0])
    out = dec.attn_paged(q, srv.cache, good, scratch)
    want, S, V = _want(q.double().cpu().view(8, heads, d), srv.k[0], srv.v[0], 2, 2991 + torch.arange(8))
    _close(out, want, S, V, d, F)


# ---------------------------------------------------------------------------------------------------- refusals

def test_what_is_refused(dev, dec):
    from paper_2410_16144_amd import binding as B
    heads, n, d = 4, 2, 64
    srv = Server(dec, dev, n, d, 16, [40, 40], 130)
    for b in range(2):
        srv.fill(b, 20)
    rows = srv.rows(dec, [10, 5], [2, 3])
    q = torch.randn((5, heads * d), generator=srv.g).to(dev)
    kv = torch.randn((5, 2 * n * d), generator=srv.g).to(dev)
    k, v = kv[:, :n * d], kv[:, n * d:]
    scratch = dec.paged_scratch(heads, srv.cache, rows)
    table = dec.rope_table(d, srv.max_pos, dev)
    k0 = srv.cache.k.clone()
    errors = (AssertionError, TypeError, ValueError, B.BitLinearError)
    out = torch.full_like(q, -7.0)
    for bad in (dict(q=q.half()), dict(q=q[:4]), dict(q=q[:, :heads * d - 4]), dict(q=q.cpu()), dict(q=q.t().contiguous().t()), dict(q=q[:, :3 * d].contiguous()),
                dict(scratch=scratch[:-16]), dict(scratch=scratch.cpu()), dict(scratch=scratch.view(torch.int32)), dict(scratch=scratch[4:]),
                dict(out=out.to(G)), dict(out=out[:4]), dict(out=out.cpu()), dict(out=q), dict(out=torch.full((5, 2 * heads * d), -7.0, device=dev)[:, ::2]),
                dict(q=torch.zeros((5, 65 * n * d), device=dev))):
        a = dict(q=q, scratch=scratch, out=out)
        a.update(bad)
        if "q" in bad:
            a["out"] = None
        with pytest.raises(errors):
            dec.attn_paged(a["q"], srv.cache, rows, a["scratch"], out=a["out"])
    one = torch.ones(d, device=dev)
    for bad in (dict(q=q.half()), dict(q=q[:4]), dict(k=k[:, :-4]), dict(k=k.to(G)), dict(v=v.cpu()), dict(v=v[:1].expand(5, -1)), dict(q=q[:, ::2]), dict(g_q=one.to(G)),
                dict(g_k=one[:-1]), dict(g_k=one.cpu()), dict(table=table[:srv.max_pos - 1]), dict(table=table.double()), dict(table=table.cpu()), dict(q_dtype=torch.float16),
                dict(q_out=q), dict(q_out=out[:4]), dict(q_out=out.half())):
        a = dict(q=q, k=k, v=v, rows=rows, table=table, g_q=one, g_k=one)
        a.update(bad)
        with pytest.raises(errors):
            srv.cache.append(**a)
    for bad in (dict(q=q[:, :d]), dict(scratch=scratch[:-16]), dict(out=q)):
        a = dict(q=q, scratch=scratch, out=out)
        a.update(bad)
        with pytest.raises(errors):
            dec.AttentionPaged(heads, srv.cache, rows, a["q"], out=a["out"], scratch=a["scratch"]).launch()
    torch.cuda.synchronize()
    assert (out == -7.0).all() and torch.equal(srv.cache.k.view(torch.int16), k0.view(torch.int16)) and not scratch.any()
