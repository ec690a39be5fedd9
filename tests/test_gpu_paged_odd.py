"""Attention over pages where keys and values are not finite, against the formula in the extended reals.

The formula: a row that sees a score of NaN or +infinity, or only scores of -infinity, is NaN.  Of the others every weight is above zero, however small
(exp of a finite number), except where the score is -infinity: there it is zero.  So an infinite value of a weight above zero is infinite, an infinite value
of a weight of zero is NaN, infinities of both signs are NaN, and so is whatever has a NaN value, whatever its weight.

Tolerances for what is finite: test_gpu_paged.py.  Scores here are sums of products that bf16 and fp32 hold, so those bounds hold as they are.
"""
import math

import pytest

from test_gpu_paged import F, G, H, U, Server, _close, _gen, dec, dev   # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

INF, NAN = math.inf, math.nan


def formula(q, k, v, group, seen):
    """q [rows, heads, d], k, v [positions, key heads, d] in 64 bits; row i sees positions 0 .. seen[i] - 1.  The outputs; those of the finite values alone;
    S and V of every row (of what is finite)."""
    T, heads, d = q.shape
    out, S, V = torch.empty_like(q), torch.zeros((T, heads)), torch.zeros((T, heads))
    plain = torch.empty_like(q)
    sees = torch.arange(k.shape[0])[None] < torch.as_tensor(seen)[:, None]
    for h in range(heads):
        kk, vv, x = k[:, h // group], v[:, h // group], q[:, h]
        s = (x[:, None] * kk[None]).sum(-1) / math.sqrt(d)               # (0 * inf and inf - inf are NaN)
        top = s.masked_fill(~sees, -INF).amax(1, keepdim=True)
        odd = ~torch.isfinite(vv)
        clean = torch.where(odd, 0.0, vv)
        w = torch.exp(s - top).masked_fill(~sees, 0.0)
        plain[:, h] = torch.where(torch.isfinite(top), w @ clean / w.sum(1, keepdim=True), NAN)
        some = lambda rows, values: rows.double() @ values.double() > 0
        up, down, nan = some(sees, vv == INF), some(sees, vv == -INF), some(sees, vv.isnan()) | some(sees & (s == -INF), odd)
        o = torch.where(up, INF, torch.where(down, -INF, plain[:, h]))
        out[:, h] = torch.where(nan | (up & down) | plain[:, h].isnan(), NAN, o)
        S[:, h] = ((x.abs()[:, None] * kk.abs()[None]).sum(-1) / math.sqrt(d)).masked_fill(~sees | ~torch.isfinite(s), 0.0).amax(1)
        V[:, h] = clean.abs().amax(1)[None].expand(T, -1).masked_fill(~sees, 0.0).amax(1)
    return out, plain, S, V


def check(out, q, k, v, group, seen, dtype):
    T, heads, d = q.shape
    got = out.double().cpu().view(T, heads, d)
    want, plain, S, V = formula(q, k, v, group, seen)
    wrong = int((got.isnan() != want.isnan()).sum()), int((got[want.isinf()] != want[want.isinf()]).sum())
    assert wrong == (0, 0), "outputs that are NaN or not, of infinities, against the formula"
    finite = torch.isfinite(want)
    ok = ~plain.isnan().any(-1)                                          # (rows of NaN have no tolerance)
    if ok.any():
        rows = [torch.where(finite, got, plain)[ok][None], plain[ok][None]]
        _close(rows[0], rows[1], S[ok][None], V[ok][None].clamp(min=1e-30), d, dtype)
    return want


def _sequence(dec, dev, d, before, new, page=16, seed=0, others=()):
    """A sequence of before + new positions that holds whatever the caller puts there, and others beside it; what nobody wrote is NaN."""
    n = 2
    srv = Server(dec, dev, n, d, page, [before + new] + list(others), 200 + d + seed)
    k, v = ((torch.randn((before + new, n, d), generator=srv.g) * 0.5).to(G) for _ in range(2))
    return srv, k, v


def _attend(dec, dev, srv, q, k, v, before, new, dtype, single, group, extra=0):
    heads, d = q.shape[1], q.shape[2]
    srv.put(0, k, v)
    rows_of = [before] + [0] * (len(srv.k) - 1)
    for b in range(1, len(srv.k)):
        srv.fill(b, int((srv.lines[b] >= 0).sum()) * srv.page)
        rows_of[b] = srv.k[b].shape[0] - 1
    many = [new] + [1] * (len(srv.k) - 1)
    T = sum(many)
    full = torch.zeros((T + extra, heads * d))
    full[:new] = q.reshape(new, -1).float()
    full[new:T] = torch.randn((T - new, heads * d), generator=srv.g)
    full = full.to(dtype).to(dev)
    rows = srv.rows(dec, rows_of, many, single, None if single else T + extra)
    out = dec.attn_paged(full, srv.cache, rows, dec.paged_scratch(heads, srv.cache, rows))
    t = new
    for b in range(1, len(srv.k)):                                       # the company is as it would be alone
        check(out[t:t + 1], full[t:t + 1].double().cpu().view(1, heads, d), srv.k[b], srv.v[b], group, [srv.k[b].shape[0]], dtype)
        t += 1
    seen = [before + 1 + i for i in range(new)]
    return out[:new], full[:new].double().cpu().view(new, heads, d), seen


# Where the one large score stands, and where the values that are not finite do: in chunks that every row sees whole, in the last one, far in front, far behind
PLACES = [(300, 10, [250]), (300, 250, [10]), (300, 299, [5, 150]), (300, 3, [299]), (40, 39, [38]), (40, 0, [39]), (20, 19, [0]), (6000, 5900, [100, 3000]), (6000, 30, [5990]),
          (6000, 3000, [1, 5999])]


@pytest.mark.parametrize("before,large,at", PLACES)
@pytest.mark.parametrize("d", [48, 64, 128, 256])
@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("form", ["single", "many heads", "packed"])
def test_values_that_are_not_finite_beside_a_score_that_outweighs_them(dev, dec, before, large, at, d, dtype, form):
    """All weights but one underflow in 32 bits; they are above zero all the same."""
    n, group = 2, 18 if form == "many heads" else 3
    new = 3 if form == "packed" else 1
    srv, k, v = _sequence(dec, dev, d, before, new)
    k[large] = 8.0                                                       # scores of 8 * 8 * sqrt(d), the others of about 4
    for i, p in enumerate(at):
        v[p, :, i], v[p, :, d - 1 - i], v[p, 0, d // 2] = INF, -INF, NAN
        v[p, 1, 20] = INF if i % 2 else -INF
    q = torch.full((new, n * group, d), 8.0)
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, form != "packed", group)
    want = check(out, qd, srv.k[0], srv.v[0], group, seen, dtype)
    assert want.isinf().any() and want.isnan().any() and torch.isfinite(want).any()


@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("form", ["single", "packed"])
@pytest.mark.parametrize("company", [[], [9000], [4000, 100, 2000, 700, 5000, 3000, 1]])
def test_what_is_not_finite_does_not_depend_on_how_walks_are_cut(dev, dec, dtype, form, company):
    """The same sequence alone and beside others, whose lengths decide how many workgroups share its walk."""
    d, group, before, new = 128, 4, 5000, 2 if form == "packed" else 1
    srv, k, v = _sequence(dec, dev, d, before, new, page=64, others=company)
    k[4700] = 8.0
    v[40, :, 3], v[2000, :, 4], v[2500, :, 5], v[2500, :, 4] = INF, INF, NAN, -INF
    q = torch.full((new, 2 * group, d), 8.0)
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, form == "single", group)
    want = check(out, qd, srv.k[0], srv.v[0], group, seen, dtype)
    assert (want[0, :, 3] == INF).all() and want[0, :, 4:6].isnan().all() and torch.isfinite(want[0, :, :3]).all()


# A key's infinities make scores of both signs, or NaN where the query has a zero; +infinity makes its rows NaN.
@pytest.mark.parametrize("before,new,at", [(300, 1, [100]), (300, 1, [300]), (40, 1, [0, 39]), (0, 1, [0]), (6000, 1, [3000]), (300, 4, [100, 301]), (100, 70, [120]), (6000, 3, [64]),
                                           (0, 5, [2]), (0, 130, [70])])
@pytest.mark.parametrize("d", [48, 64, 128, 256])
@pytest.mark.parametrize("dtype", [F, G])
@pytest.mark.parametrize("values", ["short", "full", "tiny"])
def test_keys_that_are_not_finite(dev, dec, before, new, at, d, dtype, values):
    """Head 0 meets -infinity, head 1 +infinity, head 2 zero times infinity, head 3 infinities of both signs, head 4 does not meet it (its key head has none)."""
    srv, k, v = _sequence(dec, dev, d, before, new, seed=1)
    k[at, 0, 5] = INF
    k[at, 0, 9] = -INF
    v[at[0], 0, 7] = 3.0
    size = {"short": 1.0, "full": 1.0 + 2.0 ** -12 + 2.0 ** -20, "tiny": 2.0 ** -90}[values]
    q = torch.randn((new, 8, d), generator=srv.g).to(G).float() * size
    q[..., 5], q[..., 9] = size, 0.5 * size                              # inf and -inf: NaN
    q[:, 0, 5], q[:, 0, 9] = -size, size                                 # -inf twice
    q[:, 1, 5], q[:, 1, 9] = size, -size                                 # +inf twice
    q[:, 2, 5], q[:, 2, 9] = 0.0, size
    q[:, 3] = size
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, new == 1, 4)
    if dtype == G:
        assert torch.equal(qd, q.to(G).double())
    want = check(out, qd, srv.k[0], srv.v[0], 4, seen, dtype)
    last = want[-1]
    assert last[1:4].isnan().all() and torch.isfinite(last[4:]).all() and (torch.isfinite(last[0]).all() or before + new == len(at))


@pytest.mark.parametrize("before,new,at", [(300, 1, 100), (300, 1, 300), (6000, 1, 3000), (300, 4, 100), (300, 4, 302), (100, 70, 120), (2000, 66, 2010)])
@pytest.mark.parametrize("d", [64, 128, 256])
@pytest.mark.parametrize("dtype", [F, G])
def test_an_infinite_value_of_a_weight_of_zero(dev, dec, before, new, at, d, dtype):
    """A score of -infinity is a weight of zero: zero times an infinite value is NaN, of a finite one nothing."""
    srv, k, v = _sequence(dec, dev, d, before, new, seed=2)
    k[at, 0, 5] = INF
    v[at, 0, 7], v[at, 0, 8], v[at, 0, 9] = INF, -INF, NAN
    q = torch.randn((new, 8, d), generator=srv.g).to(G).float()
    q[..., 5] = -1.0
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, new == 1, 4)
    want = check(out, qd, srv.k[0], srv.v[0], 4, seen, dtype)
    assert want[-1, :4, 7:10].isnan().all() and torch.isfinite(want[-1, :4, :7]).all() and torch.isfinite(want[-1, 4:]).all()


@pytest.mark.parametrize("before,new", [(300, 1), (5000, 1), (300, 40), (0, 3)])
@pytest.mark.parametrize("dtype", [F, G])
def test_rows_that_see_scores_of_minus_infinity_alone(dev, dec, before, new, dtype):
    """NaN: there is no largest score to be relative to.  The other key head's rows are untouched."""
    d = 64
    srv, k, v = _sequence(dec, dev, d, before, new, seed=3)
    k[:, 0, 5] = INF
    q = torch.randn((new, 6, d), generator=srv.g).to(G).float()
    q[..., 5] = -1.0
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, new == 1, 3)
    want = check(out, qd, srv.k[0], srv.v[0], 3, seen, dtype)
    assert want[:, :3].isnan().all() and torch.isfinite(want[:, 3:]).all()


@pytest.mark.parametrize("extra", [0, 2200, 7000])
@pytest.mark.parametrize("d", [64, 96, 128])
@pytest.mark.parametrize("before,new", [(0, 65), (100, 40), (500, 130)])
def test_values_and_large_scores_in_every_form_of_the_tiles(dev, dec, d, before, new, extra):
    """A row's largest score is a late one; before it and behind it values that are not finite, some of which only later rows see."""
    srv, k, v = _sequence(dec, dev, d, before, new, seed=4)
    k[before + new // 2] = 8.0
    for i, p in enumerate((0, before + new // 4, before + new // 2 + 3, before + new - 1)):
        v[p, :, i], v[p, :, d - 1 - i], v[p, 0, 30 + i], v[p, 1, 25] = INF, -INF, NAN, INF if i % 2 else -INF
    q = torch.full((new, 6, d), 8.0)
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, G, False, 3, extra)
    check(out, qd, srv.k[0], srv.v[0], 3, seen, G)


@pytest.mark.parametrize("power", [8, 20, 29, 31, 40, 70, 110])
@pytest.mark.parametrize("heads,d,before,new", [(4, 64, 300, 1), (4, 128, 6000, 1), (4, 256, 40, 1), (36, 64, 300, 1), (4, 48, 300, 70), (4, 128, 6000, 3), (4, 256, 130, 40), (4, 64, 0, 1)])
@pytest.mark.parametrize("dtype", [F, G])
def test_scores_of_any_size(dev, dec, power, heads, d, before, new, dtype):
    """Queries of +-2^power and keys of small whole numbers: scores are exact in every order of their sums, and those below the largest by a step or more weigh less than
    exp(-2^8 / 16).  What is left are sums of equal weights: divisions and sums, 40 u of the largest value, and bf16's roundings of weights and outputs.  In the tiles
    a maximum below 2^10 (in exponents of two) is rounded, by 2^-15 at most; weights relative to two such ones are off by 2^-14 ln 2, outputs by twice that."""
    srv, k, v = _sequence(dec, dev, d, before, new, seed=5)
    k = torch.randint(-3, 4, k.shape, generator=srv.g).to(G)
    if before > 100:
        k[before - 60], k[70] = k[3], k[3]                               # (equal scores far apart)
    q = (torch.randint(0, 2, (new, heads, d), generator=srv.g) * 2 - 1) * 2.0 ** power
    q[..., 0, :] = torch.where(k[min(3, before), 0] < 0, -1.0, 1.0) * 2.0 ** power
    out, qd, seen = _attend(dec, dev, srv, q, k, v, before, new, dtype, new == 1, heads // 2)
    want, plain, S, V = formula(qd, srv.k[0], srv.v[0], heads // 2, seen)
    got = out.double().cpu().view_as(want)
    assert torch.isfinite(got).all()
    worst = ((got - want).abs().amax(-1) / V).max().item()
    tiles = new > 1 or heads // 2 > 16
    assert worst <= (2 * H if dtype == G else 0) + 40 * U + (2.0 ** -13 if tiles and power == 8 else 0)


@pytest.mark.parametrize("heads,new,before", [(4, 1, 60000), (2, 9, 20000), (34, 1, 20000)])
@pytest.mark.parametrize("dtype", [F, G])
def test_what_nobody_wrote_costs_nothing(dev, dec, heads, new, before, dtype):
    """Columns of an operand that have no row do not see what lies behind the last position: a walk is not repeated because of it.  (It took twice as long.)"""
    d = 128
    srv, k, v = _sequence(dec, dev, d, before, new, page=64, seed=6)
    srv.put(0, k, v)
    q = (torch.randn((new, heads * d), generator=srv.g)).to(dtype).to(dev)
    rows = srv.rows(dec, [before], [new], new == 1)
    scratch = dec.paged_scratch(heads, srv.cache, rows)
    last, inside = int(srv.lines[0, (before + new - 1) // 64]), (before + new - 1) % 64 + 1
    assert inside % 32                                                   # the last chunk ends inside a page

    def time(fill):
        for pool in (srv.cache.k, srv.cache.v):
            pool[last, :, inside:] = fill
        best = math.inf
        for _ in range(15):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            for _ in range(20):
                out = dec.attn_paged(q, srv.cache, rows, scratch)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best, out
    time(0.0)
    (zeros, a), (nans, b) = time(0.0), time(NAN)
    assert torch.equal(a, b)
    assert nans <= 1.2 * zeros, (nans, zeros)


@pytest.mark.parametrize("power", [12, 20, 33])
@pytest.mark.parametrize("d", [4, 12, 48, 64, 128, 256])
@pytest.mark.parametrize("before,new,heads", [(0, 14, 32), (3, 60, 8), (40, 1, 8), (40, 1, 36), (700, 9, 4)])
@pytest.mark.parametrize("dtype", [F, G])
def test_equal_scores_weigh_the_same(dev, dec, power, d, before, new, heads, dtype):
    """Every key makes the same score, a small one of large terms that cancel: exact in every order of its sums, if nothing is added to them that is not there.  The outputs are the
    means of what the rows see, to the roundings of test_scores_of_any_size."""
    srv, k, v = _sequence(dec, dev, d, before, new, seed=7)
    k = torch.zeros((before + new, 2, d))
    for j in range(before + new):
        for h in range(2):
            one, two, three = torch.randperm(d, generator=srv.g)[:3].tolist()
            k[j, h, one] = int(torch.randint(1, 121, (1,), generator=srv.g))
            k[j, h, two], k[j, h, three] = -k[j, h, one], -1.0
    q = torch.full((new, heads, d), 2.0 ** power)
    out, qd, seen = _attend(dec, dev, srv, q, k.to(G), v, before, new, dtype, new == 1, heads // 2)
    want, plain, S, V = formula(qd, srv.k[0], srv.v[0], heads // 2, seen)
    got = out.double().cpu().view_as(want)
    worst = ((got - want).abs().amax(-1) / V).max().item()
    assert worst <= (2 * H if dtype == G else 0) + 40 * U
