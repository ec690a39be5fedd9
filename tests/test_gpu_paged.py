"""The paged cache (bl_paged_append) and the attention over it (bl_attn_paged) against plain 64-bit formulas.

Whatever the call does not own is NaN: pages of nobody, the rest of a sequence's last page, positions that are written later.

Tolerances, u = 2^-24 (fp32) and h = 2^-8 (bf16, half a step relative to the value):
  * append: the sum of squares is off by fewer than 16 + 4 roundings of its own size (its square root halves that), the quotient, square root and
    products by six more, the rotation by three relative to the pair's length: below 30 u of the pair's length; stored or written in bf16: h of the value more.
  * scores: exact products in 3 head_dim (fp32) or head_dim (bf16) additions, each rounded by at most u S, S = sum |q k| / sqrt(head_dim): their
    root mean square sum is below sqrt(head_dim) u S, five times that is E.  A weight is off by E of itself, so the output by at most 2 E V, V the largest
    |value| that the row sees; exp2, its argument (relative to the largest score S), sums and the division: below (40 + 4 S) u V.
  * bf16: a weight's own rounding moves the output by at most h V, its own rounding by h of itself: 2 h V in all.
    Over a whole output with independent values, the roundings' root mean squares: each h / sqrt(3) of the output, together below 0.82 h.
"""
import math

import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
U, H = 2.0 ** -24, 2.0 ** -8
F, G = torch.float32, torch.bfloat16


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def dec():
    from paper_2410_16144_amd import binding, decoder
    binding.lib()
    return decoder


def _gen(seed):
    return torch.Generator().manual_seed(seed)


class Server:
    """Sequences in pages of a pool, and what they hold in 64 bits: k, v [positions, key heads, dim] per sequence."""

    def __init__(self, dec, dev, n, d, page, capacities, seed=0, spare=3, unowned=math.nan):
        self.n, self.d, self.page, self.dev, self.g = n, d, page, dev, _gen(seed)
        need = [-(-c // page) for c in capacities]
        pages = sum(need) + spare
        order = torch.randperm(pages, generator=self.g).to(torch.int32)
        self.lines = torch.full((len(need), max(need) + 1), -5, dtype=torch.int32)
        at = 0
        for b, m in enumerate(need):
            self.lines[b, :m] = order[at:at + m]
            at += m
        self.max_pos = max(need) * page
        self.cache = dec.PagedCache(n, d, page, pages, dev)
        self.cache.k.fill_(unowned)
        self.cache.v.fill_(unowned)
        self.k = [torch.zeros((0, n, d), dtype=torch.float64) for _ in need]
        self.v = [torch.zeros((0, n, d), dtype=torch.float64) for _ in need]

    def put(self, b, k, v):
        """Rows k, v [rows, n, d] (values of bf16) behind sequence b's."""
        p0 = self.k[b].shape[0]
        self.k[b], self.v[b] = torch.cat([self.k[b], k.double()]), torch.cat([self.v[b], v.double()])
        if not k.shape[0]:
            return
        at = torch.arange(p0, p0 + k.shape[0])
        page = self.lines[b][at // self.page].long().to(self.dev)
        slot = (at % self.page).to(self.dev)
        for pool, x in ((self.cache.k, k), (self.cache.v, v)):
            full = torch.zeros((x.shape[0], self.n, pool.shape[3]), dtype=G)
            full[..., :self.d] = x.to(G)
            pool[page, :, slot] = full.to(self.dev)

    def fill(self, b, rows):
        k, v = (torch.randn((rows, self.n, self.d), generator=self.g).to(G) for _ in range(2))
        self.put(b, k, v)

    def rows(self, dec, before, new, single=False, total=None, lines=None, max_pos=None):
        pos = torch.tensor(before, dtype=torch.int32, device=self.dev)
        lines = (self.lines if lines is None else lines).to(self.dev)
        max_pos = self.max_pos if max_pos is None else max_pos
        if single:
            return dec.PagedRows(lines, pos, max_pos)
        start = torch.tensor(np.concatenate([[0], np.cumsum(new)]), dtype=torch.int32, device=self.dev)
        return dec.PagedRows(lines, pos, max_pos, start=start, rows=int(sum(new) if total is None else total))


def _want(q, k, v, group, seen):
    """q [rows, heads, d], k, v [positions, key heads, d], all in 64 bits; row i sees positions 0 .. seen[i] - 1.  Outputs, S and V of every row."""
    out, S, V = torch.empty_like(q), torch.empty(q.shape[:2]), torch.empty(q.shape[:2])
    n = torch.arange(k.shape[0])
    for h in range(q.shape[1]):
        kk, vv = k[:, h // group], v[:, h // group]
        beyond = n[None] >= seen[:, None]
        s = (q[:, h] @ kk.t() / math.sqrt(q.shape[2])).masked_fill(beyond, -math.inf)
        w = torch.softmax(s, 1)
        out[:, h] = w @ vv
        S[:, h] = (q[:, h].abs() @ kk.abs().t() / math.sqrt(q.shape[2])).masked_fill(beyond, 0).amax(1)
        V[:, h] = vv.abs().amax(1)[None].expand(q.shape[0], -1).masked_fill(beyond, 0).amax(1)
    return out, S, V


def _close(got, want, S, V, d, dtype):
    got = got.double().cpu().view_as(want)
    assert torch.isfinite(got).all()
    E = 5 * math.sqrt(d) * U * S
    bound = (2 * E + (40 + 4 * S) * U + (2 * H if dtype == G else 0)) * V
    worst = ((got - want).abs().amax(-1) / bound).max().item()
    assert worst <= 1, worst
    if got.numel() >= 1000:
        rel = ((got - want).norm() / want.norm()).item()
        assert rel <= (0.82 * H if dtype == G else 0) + 2 * (E.max().item() / 5 + 12 * U) , rel


def _queries(g, T, heads, d, dtype, dev, size=1.5):
    return (torch.randn((T, heads * d), generator=g) * size).to(dtype).to(dev)


def _attend(dec, dev, heads, n, d, page, before, new, dtype, seed, single=False, extra=0, capacity=None, scratch=None, unowned=math.nan, max_pos=None):
    srv = Server(dec, dev, n, d, page, [max(1, b + m) for b, m in zip(before, new)] if capacity is None else capacity, seed, unowned=unowned)
    for b in range(len(before)):
        srv.fill(b, before[b] + new[b])
    T = sum(new) + extra
    q = _queries(srv.g, T, heads, d, dtype, dev)
    out = torch.full((T, heads * d), -7.0, dtype=dtype, device=dev)
    rows = srv.rows(dec, before, new, single, T, max_pos=max_pos)
    scratch = dec.paged_scratch(heads, srv.cache, rows) if scratch is None else scratch
    got = dec.attn_paged(q, srv.cache, rows, scratch, out=out)
    assert got.data_ptr() == out.data_ptr()
    t = 0
    for b in range(len(before)):
        if new[b]:
            want, S, V = _want(q[t:t + new[b]].double().cpu().view(new[b], heads, d), srv.k[b], srv.v[b], heads // n, before[b] + 1 + torch.arange(new[b]))
            _close(out[t:t + new[b]], want, S, V, d, dtype)
        t += new[b]
    assert (out[t:] == -7.0).all()                                  # rows of nobody
    assert not scratch[:1 << 16].any()                              # the counters, as they were
    return srv, q, rows, scratch, out


# ---------------------------------------------------------------------------------------------------- attention

SHAPES = [(4, 4, 64), (3, 1, 128), (8, 2, 128), (4, 2, 96), (2, 2, 120), (6, 2, 48), (4, 4, 100), (3, 3, 4), (10, 5, 36), (14, 2, 128), (4, 2, 256), (2, 1, 192),
          (5, 5, 160), (16, 1, 32), (34, 2, 64), (64, 1, 80)]


@pytest.mark.parametrize("heads,n,d", SHAPES)
@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("page,before", [(16, [0]), (16, [15, 31, 0]), (64, [63, 64, 65, 1]), (32, [700, 5, 256]), (256, [0, 300])])
def test_one_token_each(dev, dec, heads, n, d, dtype, page, before):
    _attend(dec, dev, heads, n, d, page, before, [1] * len(before), dtype, 10 * d + page, single=True)


@pytest.mark.parametrize("heads,n,d", SHAPES)
@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("page,before,new", [(16, [0], [1]), (16, [0, 5], [33, 7]), (64, [0, 100, 0, 3], [130, 1, 0, 64]), (32, [500], [5]), (64, [37, 0], [65, 129])])
def test_packed_sequences(dev, dec, heads, n, d, dtype, page, before, new):
    _attend(dec, dev, heads, n, d, page, before, new, dtype, 20 * d + page, extra=3)


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("heads,n,d,before,new", [
    (8, 1, 128, [20011], None), (4, 4, 64, [9000, 17, 3000], None), (16, 2, 256, [5000], None), (40, 2, 64, [6000, 1], None), (2, 1, 48, [30000], None),
    (1, 1, 4, [9000], None), (4, 2, 128, [7001], [5]), (4, 4, 128, [3000, 4000, 0], [20, 3, 300]), (2, 2, 256, [2500], [70]), (8, 8, 64, [0], [1500]),
    (8, 2, 128, [0, 0, 900], [700, 300, 513])])
def test_long_walks(dev, dec, dtype, heads, n, d, before, new):
    """Walks that several workgroups share, as single tokens and as few and many rows behind a cache."""
    _attend(dec, dev, heads, n, d, 64, before, new or [1] * len(before), dtype, 3 * d + before[0], single=new is None, unowned=3.0e38)


@pytest.mark.parametrize("dtype", [F, G])
def test_many_sequences(dev, dec, dtype):
    """More sequences than lanes, of every length, some without rows."""
    r = np.random.default_rng(5)
    before = [int(x) for x in r.integers(0, 200, 300)]
    _attend(dec, dev, 4, 2, 64, 16, before, [1] * 300, dtype, 1, single=True)
    _attend(dec, dev, 4, 2, 64, 16, before, [int(x) for x in r.integers(0, 4, 300)], dtype, 2, extra=70)


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("capacity", [512, 200000])
def test_the_bound_on_positions_moves_no_result(dev, dec, dtype, capacity):
    """max_pos decides how many workgroups may share a walk, not what comes out."""
    for new in ([1, 1], [40, 3]):
        _attend(dec, dev, 4, 2, 128, 64, [400, 100], new, dtype, 9, single=new == [1, 1], capacity=[capacity, 512], max_pos=capacity if capacity > 512 else 448)


# ---------------------------------------------------------------------------------------------------- what takes no part

@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("single", [True, False])
def test_sequences_that_take_no_part(dev, dec, dtype, single):
    """Negative and too far positions, and rows that are not there: outputs and pools as they were, the others right."""
    heads, n, d = 4, 2, 64
    srv = Server(dec, dev, n, d, 16, [64] * 5, 3)
    for b in range(5):
        srv.fill(b, 40)
    before, new = [39, -1, 63, 64, 20], [1, 1, 1, 1, 1] if single else [3, 4, 2, 1, 20]
    before[0] -= 0 if single else 2
    T = sum(new)
    q = _queries(srv.g, T, heads, d, dtype, dev)
    rows = srv.rows(dec, before, new, single, T)
    max_pos = 64
    out = torch.full_like(q, -7.0)
    dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows), out=out)
    t = 0
    for b in range(5):
        if 0 <= before[b] <= max_pos - new[b] and before[b] + new[b] <= 40:
            want, S, V = _want(q[t:t + new[b]].double().cpu().view(new[b], heads, d), srv.k[b], srv.v[b], 2, before[b] + 1 + torch.arange(new[b]))
            _close(out[t:t + new[b]], want, S, V, d, dtype)
        elif not 0 <= before[b] <= max_pos - new[b]:
            assert (out[t:t + new[b]] == -7.0).all(), b
        t += new[b]


@pytest.mark.parametrize("start", [[0, 3, -1, 5, 8], [0, 3, 9, 9, 8], [4, 2, 2, 8, 8], [0, 0, 0, 0, 0], [8, 8, 8, 8, 8], [0, 2147483647, -2147483648, 5, 8]])
def test_starts_that_say_nothing_of_use(dev, dec, start):
    """Rows outside the call and falling starts: nothing outside the outputs is touched, and what a sound sequence owns alone is right."""
    heads, n, d = 4, 2, 64
    srv = Server(dec, dev, n, d, 16, [64] * 4, 4)
    for b in range(4):
        srv.fill(b, 60)
    q = _queries(srv.g, 8, heads, d, F, dev)
    rows = dec.PagedRows(srv.lines.to(dev), torch.tensor([5, 9, 0, 20], dtype=torch.int32, device=dev), 64,
                         start=torch.tensor(start, dtype=torch.int32, device=dev), rows=8)
    guard = torch.full((24, heads * d), -7.0, device=dev)
    k0, v0 = srv.cache.k.clone(), srv.cache.v.clone()
    dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows), out=guard[8:16])
    assert (guard[:8] == -7).all() and (guard[16:] == -7).all()
    x = torch.randn((8, (heads + 2 * n) * d), generator=srv.g).to(dev)
    guard.fill_(-7.0)
    srv.cache.append(x[:, :heads * d], x[:, heads * d:(heads + n) * d], x[:, (heads + n) * d:], rows, None, q_out=guard[8:16])
    assert (guard[:8] == -7).all() and (guard[16:] == -7).all()
    mine = torch.zeros(srv.cache.pages, dtype=torch.bool)
    mine[srv.lines[srv.lines >= 0].long()] = True
    assert torch.equal(srv.cache.k[~mine.to(dev)].view(torch.int16), k0[~mine.to(dev)].view(torch.int16))
    assert torch.equal(srv.cache.v[~mine.to(dev)].view(torch.int16), v0[~mine.to(dev)].view(torch.int16))


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("bad", [-1, 1 << 20, 2147483647, -2147483648])
@pytest.mark.parametrize("single", [True, False])
def test_pages_that_are_not_there(dev, dec, dtype, bad, single):
    heads, n, d = 4, 2, 64
    srv = Server(dec, dev, n, d, 16, [400, 400, 400], 6)
    for b in range(3):
        srv.fill(b, 390)
    lines = srv.lines.clone()
    lines[1, 3] = bad                                   # positions 48 .. 63 of sequence 1
    lines[2, 20] = bad                                  # behind the last position that is asked for
    before, new = ([300, 300, 300], [1, 1, 1]) if single else ([0, 10, 200], [30, 250, 100])
    q = _queries(srv.g, sum(new), heads, d, dtype, dev)
    rows = srv.rows(dec, before, new, single, lines=lines)
    out = dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows))
    t = 0
    for b in range(3):
        got = out[t:t + new[b]]
        if b == 1:
            first = max(0, 48 - before[b])
            assert got[first:].isnan().all()
        else:
            want, S, V = _want(q[t:t + new[b]].double().cpu().view(new[b], heads, d), srv.k[b], srv.v[b], 2, before[b] + 1 + torch.arange(new[b]))
            _close(got, want, S, V, d, dtype)
        t += new[b]


# ---------------------------------------------------------------------------------------------------- numbers that are not finite

@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("heads,n,d", [(2, 2, 64), (8, 2, 128), (2, 1, 48), (3, 1, 256)])
@pytest.mark.parametrize("before,new", [(0, 3), (30, 5), (100, 150), (0, 65), (500, 130)])
def test_what_a_row_does_not_see_has_no_part_in_it(dev, dec, dtype, heads, n, d, before, new):
    """The last token's key and value are not finite: rows before it are as if they were not there, its own row is what the formula makes of it."""
    srv = Server(dec, dev, n, d, 16, [before + new], 8)
    srv.fill(0, before + new - 1)
    k, v = torch.randn((1, n, d), generator=srv.g).to(G), torch.randn((1, n, d), generator=srv.g).to(G)
    v[0, :, 0], v[0, :, 1], v[0, :, 2] = math.inf, -math.inf, math.nan
    srv.put(0, k, v)
    q = _queries(srv.g, new, heads, d, dtype, dev)
    rows = srv.rows(dec, [before], [new])
    scratch = dec.paged_scratch(heads, srv.cache, rows)
    out = dec.attn_paged(q, srv.cache, rows, scratch).cpu().view(new, heads, d)
    qd, seen = q.double().cpu().view(new, heads, d), before + 1 + torch.arange(new)
    if new > 1:
        want, S, V = _want(qd[:-1], srv.k[0][:-1], srv.v[0][:-1], heads // n, seen[:-1])
        _close(out[:-1], want, S, V, d, dtype)
    last = out[-1]
    assert (last[:, 0] == math.inf).all() and (last[:, 1] == -math.inf).all() and last[:, 2].isnan().all()
    clean = srv.v[0].clone()
    clean[-1, :, :3] = 0
    want, S, V = _want(qd[-1:], srv.k[0], clean, heads // n, seen[-1:])
    _close(last[None, :, 3:], want[..., 3:], S, V, d, dtype)
    # and a key that is not finite
    for bad in (math.inf, math.nan):
        srv.cache.k[srv.lines[0, (before + new - 1) // 16].item(), :, (before + new - 1) % 16, 3] = bad
        again = dec.attn_paged(q, srv.cache, rows, scratch).cpu().view(new, heads, d)
        assert torch.equal(again[:-1], out[:-1])
        if math.isnan(bad):
            assert again[-1].isnan().all()


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("new", [1, 40])
def test_a_query_that_is_not_finite_is_its_own_rows_matter(dev, dec, dtype, new):
    srv, q, rows, scratch, out = _attend(dec, dev, 4, 2, 64, 16, [300], [new], dtype, 11)
    q2 = q.clone()
    q2[0, 64 + 5] = math.nan                            # head 1 of the first row
    got = dec.attn_paged(q2, srv.cache, rows, scratch)
    assert got[0, 64:128].isnan().all()
    got[0, 64:128] = out[0, 64:128]
    assert torch.equal(got, out)


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("before,new", [(700, 1), (100, 60)])
def test_scores_of_extreme_sizes(dev, dec, dtype, before, new):
    """One key's score far above the others', and scores far below zero throughout."""
    heads, n, d = 4, 2, 64
    for size in (-40.0, 40.0):
        srv = Server(dec, dev, n, d, 16, [before + new], 12)
        k, v = torch.ones((before + new, n, d)).to(G), torch.randn((before + new, n, d), generator=srv.g).to(G)
        k[before // 2] = 2.0
        srv.put(0, k, v)
        q = torch.full((new, heads * d), size, dtype=dtype, device=dev)      # scores of 8 * size, and one of 16 * size
        rows = srv.rows(dec, [before], [new])
        out = dec.attn_paged(q, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows))
        want, S, V = _want(q.double().cpu().view(new, heads, d), srv.k[0], srv.v[0], 2, before + 1 + torch.arange(new))
        _close(out, want, S, V, d, dtype)


# ---------------------------------------------------------------------------------------------------- calls one after the other

@pytest.mark.parametrize("dtype", [F, G])
def test_one_scratch_for_calls_of_all_kinds(dev, dec, dtype):
    """Few and many sequences, single and packed, on one scratch; every call again gives the same bits."""
    srv = Server(dec, dev, 2, 64, 16, [5000, 300] + [50] * 70, 14)
    for b, m in enumerate([5000, 300] + [50] * 70):
        srv.fill(b, m)
    calls = []
    for before, new, single in (([4000, 200], [1, 1], True), ([4000, 299] + [40] * 70, [1] * 72, True), ([4500, 0], [7, 200], False),
                                ([3000, 100] + [10] * 70, [3, 1] + [2] * 70, False), ([0], [900], False), ([4999], [1], True)):
        lines = srv.lines[:len(before)]
        q = _queries(srv.g, sum(new), 8, 64, dtype, dev)
        calls.append((before, new, q, srv.rows(dec, before, new, single, lines=lines.contiguous())))
    scratch = max((dec.paged_scratch(8, srv.cache, c[3]) for c in calls), key=lambda t: t.numel())
    first = []
    for before, new, q, rows in calls + calls[::-1]:
        out = dec.attn_paged(q, srv.cache, rows, scratch)
        i = len(first)
        first.append(out)
        if i >= len(calls):
            assert torch.equal(out, first[2 * len(calls) - 1 - i])
            continue
        t = 0
        for b in range(len(before)):
            want, S, V = _want(q[t:t + new[b]].double().cpu().view(new[b], 8, 64), srv.k[b], srv.v[b], 4, before[b] + 1 + torch.arange(new[b]))
            _close(out[t:t + new[b]], want, S, V, 64, dtype)
            t += new[b]


def test_offsets_beyond_32_bits(dev, dec):
    """Pools of more than 2^32 bytes and elements; the sequence's pages at both ends."""
    n, d, page = 8, 128, 64
    pages = (1 << 32) // (n * d * page) + 40
    cache = dec.PagedCache(n, d, page, pages, dev)
    g = _gen(15)
    order = torch.tensor([pages - 1, 0, pages - 2, 1, pages // 2, pages - 3], dtype=torch.int32)
    srv = Server.__new__(Server)
    srv.n, srv.d, srv.page, srv.dev, srv.g, srv.cache, srv.max_pos = n, d, page, dev, g, cache, 6 * page
    srv.lines, srv.k, srv.v = order[None], [torch.zeros((0, n, d), dtype=torch.float64)], [torch.zeros((0, n, d), dtype=torch.float64)]
    srv.fill(0, 370)
    for before, new, single in ((369, 1, True), (300, 70, False)):
        q = _queries(g, new, 16, d, G, dev)
        rows = srv.rows(dec, [before], [new], single)
        out = dec.attn_paged(q, cache, rows, dec.paged_scratch(16, cache, rows))
        want, S, V = _want(q.double().cpu().view(new, 16, d), srv.k[0], srv.v[0], 2, before + 1 + torch.arange(new))
        _close(out, want, S, V, d, G)
    x = torch.randn((1, (16 + 2 * n) * d), generator=g).to(dev)
    rows = srv.rows(dec, [383], [1], True)
    cache.append(x[:, :16 * d], x[:, 16 * d:24 * d], x[:, 24 * d:], rows, None)
    assert torch.equal(cache.k[pages - 3, :, 63, :d].flatten(), x[0, 16 * d:24 * d].to(G)) and torch.equal(cache.v[pages - 3, :, 63, :d].flatten(), x[0, 24 * d:].to(G))


# ---------------------------------------------------------------------------------------------------- append

def _append_want(x, heads, d, gamma, eps, angles):
    """x [rows, heads * d] in 64 bits; angles [rows, d / 2, 2] or None.  The values, and every element's pair's length."""
    y = x.view(-1, heads, d)
    if gamma is not None:
        y = y * gamma / torch.sqrt((y * y).mean(-1, keepdim=True) + eps)
    a, b = y[..., :d // 2], y[..., d // 2:]
    size = torch.cat([torch.hypot(a, b)] * 2, -1)
    if angles is not None:
        c, s = angles[:, None, :, 0], angles[:, None, :, 1]
        y = torch.cat([a * c - b * s, a * s + b * c], -1)
    return y, size


@pytest.mark.parametrize("heads,n,d", [(4, 4, 64), (8, 2, 128), (3, 1, 100), (2, 2, 120), (5, 5, 36), (1, 1, 4), (6, 3, 256), (7, 7, 160), (2, 1, 252), (3, 3, 48)])
@pytest.mark.parametrize("dtype,q_dtype", [(F, F), (F, G), (G, G), (G, F)])
@pytest.mark.parametrize("normed,rotated", [(True, True), (False, True), (True, False)])
@pytest.mark.parametrize("before,new,page", [([0], [1], 16), ([17, 0, 63, 5], [40, 0, 1, 70], 32), ([3, 250], [1, 1], 64)])
def test_append(dev, dec, heads, n, d, dtype, q_dtype, normed, rotated, before, new, page):
    """Queries, keys and values at their places, every other byte of the pools as it was; projections side by side in one tensor."""
    from paper_2410_16144_amd import binding as B
    srv = Server(dec, dev, n, d, page, [b + m for b, m in zip(before, new)], 16, unowned=-7.0)
    single, extra = new == [1, 1], 0 if new == [1, 1] else 2
    T = sum(new) + extra
    x = (torch.randn((T, (heads + 2 * n) * d + 8), generator=srv.g) * torch.exp(torch.randn((T, 1), generator=srv.g))).to(dtype).to(dev)
    q, k, v = x[:, :heads * d], x[:, heads * d:(heads + n) * d], x[:, (heads + n) * d:(heads + 2 * n) * d]
    g_q, g_k = ((torch.rand(d, generator=srv.g) + 0.5).to(dev) for _ in range(2)) if normed else (None, None)
    table = dec.rope_table(d, srv.max_pos, dev) if rotated else None
    rows = srv.rows(dec, before, new, single, T)
    out = torch.full((T, heads * d), -7.0, dtype=q_dtype, device=dev)
    k0, v0 = srv.cache.k.clone(), srv.cache.v.clone()
    got = srv.cache.append(q, k, v, rows, table, g_q=g_q, g_k=g_k, eps=1e-5, q_out=out)
    assert got.data_ptr() == out.data_ptr() and (out[sum(new):] == -7.0).all()
    t = 0
    for b, (p, m) in enumerate(zip(before, new)):
        if not m:
            continue
        angles = table[p:p + m].double().cpu() if rotated else None
        at = torch.arange(p, p + m)
        page_of, slot = srv.lines[b][at // page].long().to(dev), (at % page).to(dev)
        for what, h, gamma, have, half in ((q, heads, g_q, out[t:t + m].view(m, heads, d), H if q_dtype == G else 0),
                                           (k, n, g_k, srv.cache.k[page_of, :, slot, :d], H)):
            want, size = _append_want(what[t:t + m].double().cpu(), h, d, gamma.double().cpu() if gamma is not None else None, 1e-5, angles)
            bound = 30 * U * size + half * (want.abs() + 30 * U * size) + 1e-37
            assert ((have.double().cpu() - want).abs() <= bound).all()
        assert torch.equal(srv.cache.v[page_of, :, slot, :d].flatten(), v[t:t + m].to(G).flatten())
        assert not srv.cache.k[page_of, :, slot, d:].any() and not srv.cache.v[page_of, :, slot, d:].any()
        k0[page_of, :, slot] = srv.cache.k[page_of, :, slot]
        v0[page_of, :, slot] = srv.cache.v[page_of, :, slot]
        t += m
    assert torch.equal(srv.cache.k, k0) and torch.equal(srv.cache.v, v0)
    assert B.bl_paged_width(d) == srv.cache.k.shape[3]


@pytest.mark.parametrize("bad", [-1, 1 << 20, 2147483647])
def test_append_to_a_page_that_is_not_there(dev, dec, bad):
    srv = Server(dec, dev, 2, 64, 16, [40, 40], 17, unowned=-7.0)
    lines = srv.lines.clone()
    lines[0, 1] = bad
    x = torch.randn((40, 8 * 64), generator=srv.g).to(dev)
    rows = srv.rows(dec, [10, 0], [20, 20], lines=lines)
    k0 = srv.cache.k.clone()
    out = srv.cache.append(x[:, :256], x[:, 256:384], x[:, 384:], rows, None)
    assert torch.equal(out, x[:, :256])                 # the queries are there all the same
    lost = lines.clone()
    lost[0, 1] = srv.lines[0, 1]
    for b, (p, m, t) in enumerate(((10, 20, 0), (0, 20, 20))):
        for i in range(m):
            page = int(lines[b, (p + i) // 16])
            if page != bad:
                k0[page, :, (p + i) % 16, :64] = x[t + i, 256:384].to(G).view(2, 64)
    assert torch.equal(srv.cache.k, k0)


def test_append_of_numbers_that_are_not_finite(dev, dec):
    """An infinity or NaN is its own head's matter; rows of zeros stay zeros."""
    srv = Server(dec, dev, 2, 64, 16, [16], 18, unowned=0.0)
    x = torch.randn((4, 8 * 64), generator=srv.g).to(dev)
    x[1, 64 + 3], x[2, 256] = math.nan, math.inf        # head 1 of row 1's queries, key head 0 of row 2
    x[3] = 0
    one = torch.ones(64, device=dev)
    rows = srv.rows(dec, [0], [4])
    out = srv.cache.append(x[:, :256], x[:, 256:384], x[:, 384:], rows, dec.rope_table(64, 16, dev), g_q=one, g_k=one)
    bad = out.view(4, 4, 64).isnan().any(-1).cpu()
    assert bad.tolist() == [[False] * 4, [False, True, False, False], [False] * 4, [False] * 4] and not out[3].any()
    page = int(srv.lines[0, 0])
    bad = srv.cache.k[page].isnan().any(-1).cpu()
    assert bad[0, 2] and bad.sum() == 1 and not srv.cache.k[page, :, 3].any()
