"""The attention over 8-bit caches where values and scores span many orders of magnitude, every (row, head) judged by what it weighs itself.

Reference: softmax in 64 bits over what the cache stands for.  Tolerance of one (row, head), u = 2^-24.  Let p be its exact weights (they add up
to 1), V_j the largest |value| of position j, B = sum p_j V_j: rows that a query may not see, or that it gives no weight, are not in it.
  * scores: a query's element is off by half a step of max|q| / 8355584 and by three roundings of its rotation, together below
    4.1 u max|q|; where the lowest byte's sums are rounded to units of 256, by 128 of those steps times the key's scale more; the sums'
    conversion, two factors and the exponent's argument are 8 roundings of the score.  A score's error d_j is below
    (4.1 u max|q| sum|k_j| + 128 max|q| / 8355584 scale_j) / sqrt(dim) + 8 u |s_j|, and the output moves by at most 2 max d_j B (1.1: second order);
  * weights, the value's scale in them: off by at most 2^-22 of the largest of 64 (those of a chunk), 64 * 2^-22 B = 1.53e-5 B, or (two f16
    numbers) by 2^-22 of themselves and 2^-28 of the row's largest, with the 2200 positions here 2^-22 B + 2200 * 2^-28 B = 0.9e-5 B;
  * exp2, sums over chunks, waves and workgroups, the division: some 40 u B = 2.4e-6 B.
"""
import math

import numpy as np
import pytest

from test_gpu_kv8 import _codes, _rng, _t, dev, mods  # noqa: F401 (fixtures)

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
LOUD = 4.0      # every query's first element: a key's first element moves all of a position's scores by LOUD * k / sqrt(dim)


def _bias(dim, score):
    return score * math.sqrt(dim) / LOUD


class Case:
    """Positions that all rows share (P of them), then the rows' own: a prompt's, seen by it and those behind it, or one of each sequence."""

    def __init__(self, seed, heads, n, dim, P, M, batch):
        r = _rng(seed)
        self.heads, self.n, self.dim, self.P, self.M, self.batch = heads, n, dim, P, M, batch
        self.q = r.standard_normal((M, heads, dim)).astype(np.float32)
        self.q[..., 0] = LOUD
        self.kp, self.vp, self.k, self.v = (r.standard_normal((m, n, dim)).astype(np.float32) for m in (P, P, M, M))
        self.kp[..., 0] = self.k[..., 0] = 0

    def copy(self):
        other = Case.__new__(Case)
        other.__dict__.update({k: v.copy() if isinstance(v, np.ndarray) else v for k, v in self.__dict__.items()})
        return other

    def run(self, dec, dev):
        n, dim, P, M = self.n, self.dim, self.P, self.M
        flat = lambda x: _t(x.reshape(x.shape[0], -1), dev)  # noqa: E731
        table = torch.zeros((P + M + 1, dim // 2, 2), device=dev)
        table[..., 0] = 1.0                                   # no rotation
        past = dec.KvCache8(n, dim, P + (1 if self.batch else M), dev)
        if P:
            past.write(flat(self.kp), flat(self.vp), 0)
        if not self.batch:
            out = dec.attn_prefill8(flat(self.q), flat(self.k), flat(self.v), past, table, P)
        else:
            own = dec.KvCache8(n, dim, 2, dev, sequences=M)
            pos = torch.full((M,), P, dtype=torch.int32, device=dev)
            out = dec.Attention8(self.heads, own, flat(self.q), flat(self.k), flat(self.v), pos, table, prefix=past if P else None, prefix_len=P).launch()
        return out.cpu().numpy().astype(np.float64).reshape(M, self.heads, dim)

    def check(self, dec, dev, rows=None, got=None, groups=None):
        """Every row, or those of `rows`; got: outputs of a run with other rows that they do not see.  groups: key heads, or all."""
        got = self.run(dec, dev) if got is None else got
        stored = []
        for past, new in ((self.kp, self.k), (self.vp, self.v)):
            x = np.concatenate([past, new])
            c, s = _codes(x.reshape(x.shape[0], -1), self.dim)
            stored.append((c.astype(np.float64) * s[..., None].astype(np.float64), s.astype(np.float64)))
        (k, ks), (v, _) = stored
        worst = 0.0
        for m in sorted({m for m in (range(self.M) if rows is None else rows) if 0 <= m < self.M}):
            see = list(range(self.P)) + ([self.P + m] if self.batch else list(range(self.P, self.P + m + 1)))
            for h in range(self.heads) if self.heads <= 16 else (0, 1, self.heads // 2 + 1, self.heads - 1):
                g = h // (self.heads // self.n)
                if groups is not None and g not in groups:
                    continue
                q, kk, vv, root = self.q[m, h].astype(np.float64), k[see, g], v[see, g], math.sqrt(self.dim)
                s = kk @ q / root
                p = np.exp(s - s.max())
                p /= p.sum()
                B, most = p @ np.abs(vv).max(1), np.abs(q).max()
                d = (4.1 * 2.0 ** -24 * most * np.abs(kk).sum(1) + 128 * most / 8355584 * ks[see, g]) / root + 8 * 2.0 ** -24 * np.abs(s)
                bound = (2.2 * d.max() + 64 * 2.0 ** -22 + 2.0 ** -20 + 40 * 2.0 ** -24) * B
                assert np.isfinite(got[m, h]).all(), (m, h)
                off = np.abs(got[m, h] - p @ vv).max()
                assert off <= bound, (m, h, off / max(B, 1e-300), bound / max(B, 1e-300))
                worst = max(worst, off / max(bound, 1e-300))
        return worst


# heads, key heads, head size, shared positions, rows, a batch behind a prefix: every form of the launches
FORMS = {
    "token": (4, 2, 64, 700, 1, False),
    "token of a batch": (3, 3, 96, 0, 5, True),
    "token, split": (2, 1, 128, 9000, 1, True),
    "rows": (2, 2, 128, 500, 6, False),
    "rows of many heads": (300, 300, 64, 70, 3, False),
    "rows in eights": (8, 2, 96, 300, 2, False),
    "rows behind a prefix": (4, 4, 64, 900, 3, True),
    "tiles": (2, 2, 96, 61, 70, False),
    "tiles, split": (3, 3, 128, 2100, 40, False),
    "tiles, shared heads": (10, 2, 120, 30, 50, False),
    "tiles of 256": (2, 1, 256, 100, 45, False),
    "two tiles": (64, 64, 64, 0, 560, False),
    "two tiles, folded": (130, 130, 32, 20, 520, False),
    "four tiles, folded": (130, 130, 32, 20, 900, False),
    "prefix in tiles": (4, 4, 64, 1200, 20, True),
    "prefix in tiles, shared heads": (16, 2, 128, 333, 9, True),
    "prefix in tiles, own rows apart": (64, 64, 32, 150, 34, True),
}


def _make(form, seed):
    heads, n, dim, P, M, batch = FORMS[form]
    return Case(seed, heads, n, dim, P, M, batch)


def _some(c):
    """Rows worth a look where all of them are too many."""
    return None if c.M * c.heads <= 100 else (0, 1, 15, 31, 32, 33, c.M // 2, c.M - 33, c.M - 2, c.M - 1)


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][4] > 1])
@pytest.mark.parametrize("factor", [1.0, 2.0 ** 12, 2.0 ** 20, 2.0 ** 30, 2.0 ** 60])
def test_a_large_value_that_others_do_not_see(dev, mods, form, factor):
    """The last token's value (of a batch: the last sequence's) is `factor` times as large: no other row is any the worse for it."""
    c = _make(form, 31000)
    c.v[-1] *= np.float32(factor)
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][3] > 0])
@pytest.mark.parametrize("factor", [2.0 ** 12, 2.0 ** 20, 2.0 ** 30])
def test_a_large_value_without_weight(dev, mods, form, factor):
    """A position that all rows see and none gives weight (e^-60 of the others')."""
    c = _make(form, 32000)
    for at in (0, c.P // 2, c.P - 1):
        c.vp[at] *= np.float32(factor)
        c.kp[at, :, 0] = _bias(c.dim, -60.0)
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][3] > 0])
@pytest.mark.parametrize("factor", [1.0, 2.0 ** 20, 2.0 ** 40])
def test_a_large_value_that_loses_its_weight(dev, mods, form, factor):
    """What comes first weighs much for a while, until scores larger by 60 come: none of it is left."""
    c = _make(form, 33000)
    c.vp[:2] *= np.float32(factor)
    c.kp[c.P // 2:, :, 0] = _bias(c.dim, 60.0)
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][3] > 0])
@pytest.mark.parametrize("values", [(-60, 60), (60, -60), (0, 0), (80, 80), (-100, -100), (30, 20)])
@pytest.mark.parametrize("scores", [(0.0, 0.0), (-40.0, 60.0), (60.0, -40.0)])
def test_values_and_scores_that_rise_and_fall_along_the_walk(dev, mods, form, values, scores):
    """Values from 2^a to 2^b, scores from c to d, evenly along the shared positions; the rows' own as the last of them."""
    c = _make(form, 34000)
    c.vp *= np.exp2(np.linspace(*values, c.P)).astype(np.float32)[:, None, None]
    c.v *= np.float32(2.0 ** values[1])
    c.kp[..., 0] = _bias(c.dim, 1.0) * np.linspace(*scores, c.P)[:, None]
    c.k[..., 0] = _bias(c.dim, scores[1])
    if values == (30, 20):      # ... and most of them nothing at all
        c.vp[np.arange(c.P) % 7 != 3] = 0
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("seed", range(3))
def test_values_of_every_size(dev, mods, form, seed):
    """Every position's value of a size of its own between 2^-40 and 2^40, scores that spread by tens."""
    c = _make(form, 35000 + seed)
    r = _rng(36000 + seed)
    c.vp *= np.exp2(r.uniform(-40, 40, (c.P, c.n, 1))).astype(np.float32)
    c.v *= np.exp2(r.uniform(-40, 40, (c.M, c.n, 1))).astype(np.float32)
    c.kp[..., 0] = _bias(c.dim, 12.0) * r.standard_normal((c.P, c.n))
    c.k[..., 0] = _bias(c.dim, 12.0) * r.standard_normal((c.M, c.n))
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", list(FORMS))
def test_heads_of_zeros(dev, mods, form):
    """Values that are zero in a head, or up to the rows' own; keys that are zero; a query that is zero (the mean of all values)."""
    c = _make(form, 37000)
    c.vp[:, 0] = 0
    c.kp[:, -1] = 0
    c.q[0, 0] = 0
    c.check(mods[1], dev, _some(c))
    c.vp[:], c.v[:-1] = 0, 0
    c.check(mods[1], dev, _some(c))
    c.v[-1] = 0
    c.check(mods[1], dev, _some(c))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("q,k,v", [(-92, 92, 0), (92, -92, 0), (0, 0, 93), (-40, 40, -93), (-95, 90, 90)])
def test_queries_keys_and_values_of_extreme_sizes(dev, mods, form, q, k, v):
    """All of them by powers of two that leave the scores as they are, or small: the outputs are the same but for the values' power."""
    c = _make(form, 41000)
    c.q, c.k, c.v = c.q * np.float32(2.0 ** q), c.k * np.float32(2.0 ** k), c.v * np.float32(2.0 ** v)
    c.kp, c.vp = c.kp * np.float32(2.0 ** k), c.vp * np.float32(2.0 ** v)
    c.check(mods[1], dev, _some(c))


NAN, INF = float("nan"), float("inf")


@pytest.mark.parametrize("form", [f for f in FORMS if FORMS[f][4] > 1])
@pytest.mark.parametrize("which,what", [("v", INF), ("v", -INF), ("v", NAN), ("k", INF), ("k", NAN), ("kv", NAN)])
def test_rows_that_are_not_finite_and_not_seen(dev, mods, form, which, what):
    """An element of the last token's row (of a batch: of the last sequence's): every other token's output is as it was."""
    c = _make(form, 38000)
    clean = c.copy()
    for name in which:
        getattr(c, name)[-1, :, 5] = what
    last = c.M - 1
    clean.check(mods[1], dev, [m for m in (_some(c) or range(c.M)) if m != last], got=c.run(mods[1], dev))


@pytest.mark.parametrize("form", list(FORMS))
@pytest.mark.parametrize("which,what", [("v", INF), ("v", -INF), ("v", NAN), ("k", INF), ("k", -INF), ("k", NAN)])
def test_rows_that_are_not_finite_and_seen(dev, mods, form, which, what):
    """An element of a key head's row: the output of every query that sees it is NaN, whatever weight it has; all others are as they were."""
    c, dec = _make(form, 39000), mods[1]
    for at, bias in ((0, 0.0), (c.P // 2, -300.0), (c.P - 1, 10.0), (c.P + c.M // 2, 0.0)):
        if at < 0:
            continue
        own = at - c.P
        row = lambda case, name: getattr(case, name + "p")[at] if own < 0 else getattr(case, name)[own]  # noqa: B023, E731
        if bias:
            row(c, "k")[:, 0] = _bias(c.dim, bias)
        bad = c.copy()
        for name in which:
            row(bad, name)[0, 5] = what
        got = bad.run(dec, dev)
        sees = [m for m in (_some(c) or range(c.M)) if 0 <= m < c.M and (own < 0 or (m == own if c.batch else m >= own))]
        assert np.isnan(got[sees][:, :c.heads // c.n]).all()
        c.check(dec, dev, [m for m in (_some(c) or range(c.M)) if m not in sees], got=got)
        c.check(dec, dev, sees, got=got, groups=range(1, c.n))


@pytest.mark.parametrize("dim", [64, 96, 100, 252])
@pytest.mark.parametrize("what", [INF, -INF, NAN])
def test_every_writer_stores_a_row_that_is_not_finite_alike(dev, mods, dim, what):
    """Codes 0 and a scale of NaN, through write (fp32 and bf16), a prompt of few rows and of many, and a token; all other heads and rows
    as without it.  Read back, the row is NaN."""
    B, dec, ops = mods
    n, M, at = 2, 41, 17
    r = _rng(40000 + dim)
    k, v = (r.standard_normal((M, n, dim)).astype(np.float32) for _ in range(2))
    k, v = (torch.from_numpy(x).bfloat16().float().numpy() for x in (k, v))
    flat = lambda x: _t(x.reshape(len(x), -1), dev)  # noqa: E731
    table = torch.rand((M, dim // 2, 2), device=dev, generator=torch.Generator(device=dev).manual_seed(1)) + 0.5
    for e in (0, dim // 2 - 1, dim - 1):
        bad_k, bad_v = k.copy(), v.copy()
        bad_k[at, 0, e] = bad_v[at, 1, e] = what
        caches = [dec.KvCache8(n, dim, M, dev) for _ in range(5)]
        clean = dec.KvCache8(n, dim, M, dev)
        clean.write(flat(k), flat(v), 0, table)
        caches[0].write(flat(bad_k), flat(bad_v), 0, table)
        caches[1].write(flat(bad_k).bfloat16(), flat(bad_v).bfloat16(), 0, table)
        dec.attn_prefill8(flat(bad_k), flat(bad_k), flat(bad_v), caches[2], table, 0)
        for first in range(0, M, 6):
            rows = slice(first, min(first + 6, M))
            dec.attn_prefill8(flat(bad_k[rows]), flat(bad_k[rows]), flat(bad_v[rows]), caches[3], table, first)
        for m in range(M):
            x, y = flat(bad_k[m:m + 1]), flat(bad_v[m:m + 1])
            dec.Attention8(n, caches[4], x, x, y, torch.tensor([m], dtype=torch.int32, device=dev), table).launch()
        for c in caches:
            for name, head in (("k", 0), ("v", 1)):
                scale, base = getattr(c, name + "_scale")[0], getattr(clean, name + "_scale")[0]
                assert bool(torch.isnan(scale[head, at])) and int(torch.isnan(scale).sum()) == 1
                keep = torch.ones_like(scale, dtype=torch.bool)
                keep[head, at] = False
                assert torch.equal(scale[keep], base[keep])
                assert torch.equal(getattr(c, name + "_codes"), getattr(caches[0], name + "_codes"))
            for dtype in (torch.float32, torch.bfloat16):
                for got, base, head in zip(c.read(0, M, dtype), clean.read(0, M, dtype), (0, 1)):
                    got, base = got.view(M, n, dim), base.view(M, n, dim).clone()
                    assert bool(torch.isnan(got[at, head]).all())
                    base[at, head] = got[at, head] = 0
                    assert torch.equal(got, base)
        places = caches[0].k_codes[0, 0].view(-1)
        S = (dim + 15) // 16 * 16
        e_all = np.arange(S)
        key_at = 4096 * (e_all // 64) + (16 * (at % 4) + at // 4) * np.minimum(64, S - 64 * (e_all // 64)) + e_all % 64
        assert not places[torch.from_numpy(key_at).to(dev)].any() and not caches[0].v_codes[0, 1].view(-1)[torch.from_numpy(64 * e_all + at).to(dev)].any()
