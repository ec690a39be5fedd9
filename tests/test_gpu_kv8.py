"""The 8-bit key/value cache and the attention over it (bl_kv8_*, bl_attn8_*) against plain 64-bit formulas.

What the quantizer decides is compared bit for bit with the oracle's quantizer on the fp32 rotation; attention with the softmax in 64 bits
over the values that the cache stands for.  Tolerance of the attention, u = 2^-24, V the largest |value| that the row may see:
  * scores: the query is rounded to multiples of max|q| / 8355584 behind a rotation of three fp32 operations, so a score is off by at most
    (2^-24 max|q| + 3 u |q|) sum|k| / sqrt(d) + 6 roundings of its own: below 4e-6 for the values drawn here, and so is a weight's relative
    error; the outputs move by at most twice that, 8e-6 V;
  * weights (with the value's scale in them): off by at most half a step, 2^-22 of the chunk's largest, 64 of them in a chunk whose factors
    add up to at most 1: 64 * 2^-22 V = 1.6e-5 V if all 64 roundings fall the same way;
  * exp2, sums over chunks and workgroups, the division: some 30 u = 2e-6 V.
Together below 3e-5 V for every element (kept by construction).  Over a whole output the roundings are independent, and their root mean square
is measured against V as well (an output is smaller than V by its averaging, the roundings of 64 weights of a chunk are not): weights
sqrt(64) * 2^-22 / sqrt(3) V = 1.1e-6 V (a half step's uniform error; chunks' factors add up to at most 1), scores below 4e-6 / sqrt(3) = 2.3e-6 of
their share, which averages over rows (at most V), the rest 0.2e-6 V: below 2.6e-6 V.
"""
import math

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
THETA = 10000.0


@pytest.fixture(scope="module")
def dev():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    return torch.device("cuda:0")


@pytest.fixture(scope="module")
def mods():
    from paper_2410_16144_amd import binding, decoder, ops
    binding.lib()
    return binding, decoder, ops


def _rng(seed):
    return np.random.Generator(np.random.PCG64(seed))


def _t(a, dev):
    return torch.from_numpy(np.ascontiguousarray(a)).to(dev)


def _table(dim, n):
    a = np.arange(n, dtype=np.float64)[:, None] * THETA ** (-2.0 * np.arange(dim // 2) / dim)
    return np.stack([np.cos(a), np.sin(a)], -1).astype(np.float32)


def _rotate(x, table, dim):
    """fp32, each operation rounded; x [rows, heads * dim], table [rows, dim / 2, 2]."""
    y = x.reshape(x.shape[0], -1, 2, dim // 2)
    c, s = table[:, None, :, 0].astype(x.dtype), table[:, None, :, 1].astype(x.dtype)
    return np.stack([y[:, :, 0] * c - y[:, :, 1] * s, y[:, :, 0] * s + y[:, :, 1] * c], 2).reshape(x.shape)


def _codes(x, dim):
    """The quantizer on every (row, head): codes and scales [rows, heads, (dim)]."""
    q, a, _ = oracle.quant_act(np.ascontiguousarray(x.reshape(-1, dim)))
    return q.reshape(x.shape[0], -1, dim), a.reshape(x.shape[0], -1)


def _places(p, dim):
    """Offsets of position p's codes in a head's buffers, from the header's words."""
    S = (dim + 15) // 16 * 16
    e = np.arange(dim)
    base = p // 64 * 64 * S
    return (base + 4096 * (e // 64) + (16 * (p % 4) + p % 64 // 4) * np.minimum(64, S - 64 * (e // 64)) + e % 64, base + 64 * e + p % 64)


class Model:
    """A sequence's rows as the cache holds them."""

    def __init__(self, n, dim):
        self.n, self.dim = n, dim
        self.k, self.v = np.zeros((0, n, dim)), np.zeros((0, n, dim))

    def put(self, pos0, k, v, table=None):
        """Returns codes and scales; the rows must follow or replace."""
        k = k if table is None else _rotate(k, table, self.dim)
        got = _codes(k, self.dim) + _codes(v, self.dim)
        rows = [got[0].astype(np.float64) * got[1][..., None], got[2].astype(np.float64) * got[3][..., None]]
        self.k = np.concatenate([self.k[:pos0], rows[0], self.k[pos0 + len(k):]])
        self.v = np.concatenate([self.v[:pos0], rows[1], self.v[pos0 + len(v):]])
        return got


def _attend(q, k, v, group):
    """q [heads, dim] (rotated, 64 bits) over k, v [rows, key heads, dim]."""
    out = np.empty_like(q)
    for h in range(q.shape[0]):
        s = k[:, h // group] @ q[h] / math.sqrt(q.shape[1])
        p = np.exp(s - s.max())
        out[h] = p @ v[:, h // group] / p.sum()
    return out


def _close(got, want, v):
    got = got.astype(np.float64)
    assert np.isfinite(got).all()
    worst = np.abs(got - want).max() / np.abs(v).max()
    assert worst <= 3e-5, worst
    rms = np.sqrt(np.mean((got - want) ** 2)) / np.abs(v).max()
    assert rms <= 2.6e-6, rms


def _rows(r, M, width, spread=True):
    x = r.standard_normal((M, width))
    return (x * np.exp(0.3 * r.standard_normal((M, 1))) if spread else x).astype(np.float32)


# ---------------------------------------------------------------------------------------------------- rows in and out

SHAPES = [(3, 64), (2, 128), (1, 96), (2, 120), (3, 48), (2, 100), (1, 4), (2, 36), (1, 256), (1, 160), (2, 252), (2, 8)]


@pytest.mark.parametrize("n,dim", SHAPES)
@pytest.mark.parametrize("pos0,M", [(0, 1), (63, 2), (27, 37), (0, 64), (5, 200), (64, 64), (130, 61)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_rows_in_and_out(dev, mods, n, dim, pos0, M, dtype):
    """Codes and scales bit for bit at the header's places, every other byte as it was; read back: code * scale, rounded once."""
    B, dec, ops = mods
    r = _rng(100 * dim + pos0 + M)
    dt = getattr(torch, dtype)
    table = _table(dim, pos0 + M)
    k, v = (_t(_rows(r, M, n * dim), dev).to(dt) for _ in range(2))
    cache = dec.KvCache8(n, dim, pos0 + M + 3, dev, sequences=3)
    for t in (cache.k_codes, cache.v_codes):
        t.fill_(85)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(-7.0)
    cache.write(k, v, pos0, _t(table, dev), sequence=1)
    got = dict(k=cache.k_codes.cpu().numpy(), v=cache.v_codes.cpu().numpy())
    scales = dict(k=cache.k_scale.cpu().numpy(), v=cache.v_scale.cpu().numpy())
    codes = Model(n, dim).put(0, k.float().cpu().numpy(), v.float().cpu().numpy(), table[pos0:])
    S = (dim + 15) // 16 * 16
    for which, (name, c, s) in enumerate([("k", codes[0], codes[1]), ("v", codes[2], codes[3])]):
        want, want_s = np.full_like(got[name], 85), np.full_like(scales[name], -7.0)
        for m in range(M):
            want[1][:, _places(pos0 + m, S)[which]] = 0          # the padding dims are written as zero
            want[1][:, _places(pos0 + m, dim)[which] if S == dim else _places(pos0 + m, S)[which][:dim]] = c[m]
            want_s[1][:, pos0 + m] = s[m]
        np.testing.assert_array_equal(got[name], want)
        np.testing.assert_array_equal(scales[name].view(np.uint32), want_s.view(np.uint32))
    for out_dtype in (torch.float32, torch.bfloat16):
        rk, rv = cache.read(pos0, M, out_dtype, sequence=1)
        for have, c, s in ((rk, codes[0], codes[1]), (rv, codes[2], codes[3])):
            want = torch.from_numpy((c.astype(np.float32) * s[..., None]).reshape(M, -1)).to(out_dtype)
            assert torch.equal(have.cpu(), want)


def test_rows_that_lie_apart_and_rotated_ones(dev, mods):
    """Rows of one wider matrix (keys and values side by side), stored without a table as they are; reading one side alone."""
    B, dec, ops = mods
    n, dim, M = 2, 96, 70
    both = _t(_rows(_rng(5), M, 2 * n * dim + 3), dev)
    k, v = both[:, :n * dim], both[:, n * dim + 3:]
    a, b = (dec.KvCache8(n, dim, 100, dev) for _ in range(2))
    a.write(k, v, 11)
    b.write(k.contiguous(), v.contiguous(), 11)
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, name), getattr(b, name))
    want, _, _ = oracle.quant_act(np.ascontiguousarray(k.cpu().numpy().reshape(-1, dim)))
    got, _ = a.read(11, M)
    scale = np.abs(k.cpu().numpy().reshape(-1, dim)).max(1) / np.float32(127.0)
    np.testing.assert_array_equal(got.cpu().numpy().reshape(-1, dim), want.astype(np.float32) * scale[:, None])
    wide = torch.full((M, n * dim + 5), 3.0, device=dev)
    B.bl_kv8_read(a.args, 0, wide.data_ptr(), n * dim + 5, B.BL_F32, 0, 11, M, B.current_stream())
    assert torch.equal(wide[:, :n * dim], a.read(11, M)[1]) and bool((wide[:, n * dim:] == 3.0).all())


def test_rows_of_zeros_and_of_extreme_sizes(dev, mods):
    B, dec, ops = mods
    n, dim = 1, 64
    x = _rows(_rng(6), 6, dim)
    x[0] = 0
    x[1] *= 1e-38            # 127 / amax overflows: a row of zeros
    x[2] *= 1e-30
    x[3] *= 1e30
    x[4] = 0
    x[4, 17] = -3.0
    cache = dec.KvCache8(n, dim, 6, dev)
    cache.write(_t(x, dev), _t(x[::-1].copy(), dev), 0)
    k, v = cache.read(0, 6)
    q, a, _ = oracle.quant_act(x)
    want = q.astype(np.float32) * a[:, None]
    np.testing.assert_array_equal(k.cpu().numpy(), want)
    np.testing.assert_array_equal(v.cpu().numpy(), want[::-1])
    assert not want[:2].any() and want[4, 17] == -3.0


# ---------------------------------------------------------------------------------------------------- one token

def _filled(dec, dev, r, n, dim, max_pos, rows, table, sequences=1, first=0):
    """A cache whose sequence b has rows[b] rows, garbage everywhere else, and the models of its sequences."""
    cache = dec.KvCache8(n, dim, max_pos, dev, sequences=sequences)
    cache.k_codes.fill_(-128)
    cache.v_codes.fill_(-128)
    cache.k_scale.fill_(float("nan"))
    cache.v_scale.fill_(float("inf"))
    models = []
    for b in range(sequences):
        m = Model(n, dim)
        if rows[b]:
            k, v = _rows(r, rows[b], n * dim), _rows(r, rows[b], n * dim)
            angles = table[first:first + rows[b]]
            m.put(0, k, v, angles)
            cache.write(_t(k, dev), _t(v, dev), 0, _t(angles, dev), sequence=b)
        models.append(m)
    return cache, models


def _check_step(mods, dev, heads, cache, models, pos, table, r, prefix=None, prefix_model=None, prefix_len=0, attention=None):
    """One launch; every sequence against its formula, the caches against their models."""
    B, dec, ops = mods
    n, dim, seqs = cache.n_heads, cache.head_dim, cache.sequences
    q, k, v = _rows(r, seqs, heads * dim), _rows(r, seqs, n * dim), _rows(r, seqs, n * dim)
    out = torch.full((seqs, heads * dim), -77.0, device=dev)
    a = dec.Attention8(heads, cache, _t(q, dev), _t(k, dev), _t(v, dev), _t(np.asarray(pos, np.int32), dev), _t(table, dev), prefix=prefix,
                       prefix_len=prefix_len, out=out)
    before = [getattr(cache, x).clone() for x in ("k_codes", "v_codes", "k_scale", "v_scale")]
    a.launch()
    got = out.cpu().numpy()
    for b in range(seqs):
        at = pos[b] - prefix_len
        if not 0 <= at < cache.max_pos:
            assert (got[b] == -77.0).all()
            for x, y in zip(before, (cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale)):
                assert torch.equal(x[b].view(torch.uint8), y[b].view(torch.uint8))
            continue
        angles = table[pos[b]:pos[b] + 1]
        codes = models[b].put(at, k[b:b + 1], v[b:b + 1], angles)
        S = (dim + 15) // 16 * 16
        for which, name in enumerate(("k", "v")):
            stored, scale = getattr(cache, name + "_codes")[b].cpu().numpy(), getattr(cache, name + "_scale")[b].cpu().numpy()
            np.testing.assert_array_equal(stored[:, _places(at, S)[which]][:, :dim], codes[2 * which][0])
            assert not stored[:, _places(at, S)[which]][:, dim:].any()
            np.testing.assert_array_equal(scale[:, at], codes[2 * which + 1][0])
        kk, vv = models[b].k[:at + 1], models[b].v[:at + 1]
        if prefix_len:
            kk, vv = np.concatenate([prefix_model.k[:prefix_len], kk]), np.concatenate([prefix_model.v[:prefix_len], vv])
        qr = _rotate(q[b:b + 1].astype(np.float64), angles, dim).reshape(heads, dim)
        _close(got[b].reshape(heads, dim), _attend(qr, kk, vv, heads // n), vv)
    assert not a.scratch[:B.bl_attn8_scratch_bytes(heads, n, dim, cache.max_pos, seqs, prefix_len)].view(torch.int32)[:n * -(-seqs * heads // n // 32) * 32].any()
    return a, got


@pytest.mark.parametrize("heads,n,dim", [(3, 3, 64), (2, 2, 128), (4, 1, 96), (2, 2, 120), (6, 2, 48), (5, 1, 100), (2, 1, 4), (9, 1, 36), (16, 1, 256),
                                         (2, 2, 160), (21, 1, 64), (8, 2, 192), (12, 2, 256), (7, 1, 128)])
@pytest.mark.parametrize("pos", [0, 1, 62, 63, 64, 255, 256, 700])
def test_token_attention(dev, mods, heads, n, dim, pos):
    r = _rng(7000 + 10 * dim + pos + heads)
    table = _table(dim, pos + 5)
    cache, models = _filled(mods[1], dev, r, n, dim, pos + 5, [pos], table)
    _check_step(mods, dev, heads, cache, models, [pos], table, r)


@pytest.mark.parametrize("pos", range(0, 70))
def test_token_attention_at_every_place_of_a_chunk(dev, mods, pos):
    r = _rng(8000 + pos)
    table = _table(96, 80)
    cache, models = _filled(mods[1], dev, r, 2, 96, 80, [pos], table)
    _check_step(mods, dev, 4, cache, models, [pos], table, r)


@pytest.mark.parametrize("heads,n,dim,pos,max_pos", [(32, 32, 128, 3000, 4096), (8, 1, 128, 20001, 20002), (2, 2, 64, 70000, 70001), (1, 1, 120, 5000, 200000)])
def test_token_attention_over_many_workgroups(dev, mods, heads, n, dim, pos, max_pos):
    r = _rng(9000 + pos)
    table = _table(dim, pos + 1)
    table = np.concatenate([table, np.zeros((max_pos - pos - 1, dim // 2, 2), np.float32)])
    cache, models = _filled(mods[1], dev, r, n, dim, max_pos, [pos], table)
    _check_step(mods, dev, heads, cache, models, [pos], table, r)


# ---------------------------------------------------------------------------------------------------- several sequences

@pytest.mark.parametrize("heads,n,dim", [(3, 3, 64), (2, 2, 128), (4, 2, 96), (10, 2, 36), (20, 1, 64), (4, 1, 256)])
@pytest.mark.parametrize("prefix_len,lengths", [(0, [0, 5, 64]), (1, [0, 0]), (63, [1, 200, 0, 64, 63]), (300, [7] * 3), (257, [0, 1, 2, 3, 4, 5, 6, 7, 8]),
                                                (2000, [300, 10, 0])])
def test_sequences_behind_a_prefix(dev, mods, heads, n, dim, prefix_len, lengths):
    r = _rng(10000 + dim + prefix_len + heads)
    own = max(lengths) + 2
    table = _table(dim, prefix_len + own)
    cache, models = _filled(mods[1], dev, r, n, dim, own, lengths, table, sequences=len(lengths), first=prefix_len)
    prefix, pm = _filled(mods[1], dev, r, n, dim, prefix_len + 9, [prefix_len], table) if prefix_len else (None, [None])
    _check_step(mods, dev, heads, cache, models, [prefix_len + x for x in lengths], table, r, prefix, pm[0], prefix_len)


@pytest.mark.parametrize("prefix_len", [0, 40, 3000])
def test_sequences_that_take_no_part(dev, mods, prefix_len):
    """Positions before the prefix' end, negative ones and ones beyond the cache: output and cache stay, the others are right."""
    r = _rng(11000 + prefix_len)
    heads, n, dim, own = 4, 2, 64, 100
    lengths = [30, 50, 0, 99, 20]
    table = _table(dim, prefix_len + own)
    cache, models = _filled(mods[1], dev, r, n, dim, own, lengths, table, sequences=5, first=prefix_len)
    prefix, pm = _filled(mods[1], dev, r, n, dim, max(1, prefix_len), [prefix_len], table) if prefix_len else (None, [None])
    pos = [prefix_len + 30, prefix_len - 1, prefix_len, -2147483648, prefix_len + own]
    _check_step(mods, dev, heads, cache, models, pos, table, r, prefix, pm[0], prefix_len)
    _check_step(mods, dev, heads, cache, models, [-1] * 5, table, r, prefix, pm[0], prefix_len)
    pos = [prefix_len + x for x in lengths]
    _check_step(mods, dev, heads, cache, models, pos, table, r, prefix, pm[0], prefix_len)


def test_a_large_batch_with_shared_key_heads(dev, mods):
    r = _rng(12000)
    heads, n, dim, prefix_len, own, seqs = 8, 2, 64, 500, 90, 37
    lengths = [int(x) for x in r.integers(0, own - 1, seqs)]
    table = _table(dim, prefix_len + own)
    cache, models = _filled(mods[1], dev, r, n, dim, own, lengths, table, sequences=seqs, first=prefix_len)
    prefix, pm = _filled(mods[1], dev, r, n, dim, prefix_len, [prefix_len], table)
    _check_step(mods, dev, heads, cache, models, [prefix_len + x for x in lengths], table, r, prefix, pm[0], prefix_len)


def test_a_prefix_is_the_same_as_its_rows_in_each_cache(dev, mods):
    """Sequences behind a shared prefix against sequences that have its rows in their own caches."""
    B, dec, ops = mods
    r = _rng(13000)
    heads, n, dim, P, lengths = 4, 4, 128, 450, [0, 70, 33]
    table = _table(dim, P + 100)
    t = _t(table, dev)
    pk, pv = _t(_rows(r, P, n * dim), dev), _t(_rows(r, P, n * dim), dev)
    prefix, cache = dec.KvCache8(n, dim, P, dev), dec.KvCache8(n, dim, 100, dev, sequences=3)
    whole = dec.KvCache8(n, dim, P + 100, dev, sequences=3)
    prefix.write(pk, pv, 0, t)
    for b, m in enumerate(lengths):
        whole.write(pk, pv, 0, t, sequence=b)
        if m:
            k, v = _t(_rows(r, m, n * dim), dev), _t(_rows(r, m, n * dim), dev)
            cache.write(k, v, 0, t[P:].contiguous(), sequence=b)
            whole.write(k, v, P, t, sequence=b)
    q, k, v = (_t(_rows(r, 3, n * dim), dev) for _ in range(3))
    pos = _t(np.array([P + m for m in lengths], np.int32), dev)
    a = dec.Attention8(heads, cache, q, k, v, pos, t, prefix=prefix, prefix_len=P).launch().cpu().numpy()
    b = dec.Attention8(heads, whole, q, k, v, pos, t).launch().cpu().numpy()
    assert np.linalg.norm(a - b) <= 1e-5 * np.linalg.norm(b)   # twice the bound against 64 bits
    for i, m in enumerate(lengths):
        for x, y in zip(cache.read(m, 1, sequence=i), whole.read(P + m, 1, sequence=i)):
            assert torch.equal(x, y)


# ---------------------------------------------------------------------------------------------------- prompts

def _check_prompt(mods, dev, heads, n, dim, pos0, M, seed, max_more=3, sample=None):
    B, dec, ops = mods
    r = _rng(seed)
    table = _table(dim, pos0 + M + max_more)
    cache, models = _filled(dec, dev, r, n, dim, pos0 + M + max_more, [0, pos0], table, sequences=2)
    q, k, v = _rows(r, M, heads * dim), _rows(r, M, n * dim), _rows(r, M, n * dim)
    out = dec.attn_prefill8(_t(q, dev), _t(k, dev), _t(v, dev), cache, _t(table, dev), pos0, sequence=1).cpu().numpy()
    codes = models[1].put(pos0, k, v, table[pos0:pos0 + M])
    rk, rv = cache.read(pos0, M, sequence=1)
    np.testing.assert_array_equal(rk.cpu().numpy().reshape(M, n, dim), codes[0].astype(np.float32) * codes[1][..., None])
    np.testing.assert_array_equal(rv.cpu().numpy().reshape(M, n, dim), codes[2].astype(np.float32) * codes[3][..., None])
    assert bool(torch.isnan(cache.k_scale[0]).all()) and bool((cache.k_codes[0] == -128).all())   # the other sequence
    qr = _rotate(q.astype(np.float64), table[pos0:pos0 + M], dim).reshape(M, heads, dim)
    ms = range(M) if sample is None else sample
    want = np.stack([_attend(qr[m], models[1].k[:pos0 + m + 1], models[1].v[:pos0 + m + 1], heads // n) for m in ms])
    _close(out.reshape(M, heads, dim)[list(ms)], want, models[1].v)


@pytest.mark.parametrize("heads,n,dim", [(3, 3, 64), (2, 2, 128), (4, 2, 96), (1, 1, 120), (2, 1, 48), (3, 1, 100), (2, 2, 4), (2, 2, 36), (2, 1, 256), (1, 1, 160),
                                         (17, 1, 64)])
@pytest.mark.parametrize("pos0,M", [(0, 1), (0, 2), (5, 3), (0, 33), (61, 7), (64, 64), (30, 100), (400, 5), (1000, 16)])
def test_prompt_attention(dev, mods, heads, n, dim, pos0, M):
    _check_prompt(mods, dev, heads, n, dim, pos0, M, 14000 + dim + 7 * pos0 + M)


@pytest.mark.parametrize("heads,n,dim,pos0,M", [(8, 8, 128, 512, 300), (16, 4, 64, 0, 700), (4, 4, 96, 2000, 65), (2, 2, 128, 9000, 40), (32, 32, 128, 100, 64)])
def test_prompt_attention_longer(dev, mods, heads, n, dim, pos0, M):
    ms = sorted(set([0, 1, 31, 32, 33, M // 2, M - 2, M - 1]) & set(range(M)))
    _check_prompt(mods, dev, heads, n, dim, pos0, M, 15000 + M, sample=ms)


def test_prompt_then_tokens(dev, mods):
    """Tokens one by one behind a prompt, and the same tokens as a prompt: the same cache, the same outputs within both bounds."""
    B, dec, ops = mods
    r = _rng(16000)
    heads, n, dim, M, more = 4, 2, 96, 150, 9
    table = _t(_table(dim, M + more), dev)
    q, k, v = (_t(_rows(r, M + more, w * dim), dev) for w in (heads, n, n))
    a, b = dec.KvCache8(n, dim, M + more, dev), dec.KvCache8(n, dim, M + more, dev)
    dec.attn_prefill8(q[:M], k[:M], v[:M], a, table, 0)
    whole = dec.attn_prefill8(q, k, v, b, table, 0)
    pos = torch.zeros(1, dtype=torch.int32, device=dev)
    for m in range(M, M + more):
        pos.fill_(m)
        one = dec.Attention8(heads, a, q[m:m + 1], k[m:m + 1], v[m:m + 1], pos, table).launch()
        assert float((one - whole[m]).norm()) <= 1e-5 * float(whole[m].norm())
    for name in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert torch.equal(getattr(a, name), getattr(b, name))


@pytest.mark.parametrize("heads,n,dim,pos0,M", [(32, 32, 128, 900, 5), (3, 3, 64, 1500, 8), (2, 2, 96, 2000, 9), (8, 2, 120, 1100, 2), (4, 1, 256, 700, 2), (16, 2, 256, 300, 1),
                                                (5, 5, 128, 0, 8), (2, 2, 36, 60, 7)])
def test_prompts_of_few_rows(dev, mods, heads, n, dim, pos0, M):
    """Up to eight rows of a key head, which go without tiles, and one more."""
    _check_prompt(mods, dev, heads, n, dim, pos0, M, 61000 + pos0 + M)


@pytest.mark.parametrize("heads,n,dim,prefix_len,lengths", [(32, 32, 64, 1500, [3, 0, 80, 64, 17, 300, 1, 2] * 2), (40, 40, 64, 900, [9] * 14 + [200]), (64, 64, 64, 300, [5, 70] * 17),
                                                            (33, 33, 64, 130, [2] * 63), (32, 32, 128, 2000, [7, 100, 0, 64, 65] * 1), (64, 8, 64, 500, [10, 200] * 5),
                                                            (32, 32, 128, 1000, [30] * 8), (64, 8, 128, 0, [40] * 33), (64, 4, 64, 0, [600, 1] * 3), (96, 6, 64, 0, [70] * 43)])
def test_batches_of_many_own_walks(dev, mods, heads, n, dim, prefix_len, lengths):
    """Own walks that alone fill the device beside the prefix's walk, and more than go into one launch with it; rows in eights and sixteens by
    eight waves and by four."""
    test_sequences_behind_a_prefix(dev, mods, heads, n, dim, prefix_len, lengths)


@pytest.mark.parametrize("heads,n,dim,pos0,M", [(64, 64, 64, 0, 1000), (64, 64, 64, 33, 2080), (130, 130, 32, 10, 500), (64, 8, 128, 70, 300), (300, 300, 64, 0, 130), (256, 256, 48, 5, 65)])
def test_prompts_of_many_tiles(dev, mods, heads, n, dim, pos0, M):
    """Two and four tiles per workgroup, a workgroup's blocks from both ends, an odd number of blocks, ends inside a tile."""
    _check_prompt(mods, dev, heads, n, dim, pos0, M, 63000 + pos0 + M, sample=sorted({0, 1, 31, 32, M // 2, min(M // 2 + 33, M - 1), M - 34, M - 1}))


@pytest.mark.parametrize("form", ["token", "rows", "tiles", "prefix in tiles"])
@pytest.mark.parametrize("what", [float("nan"), float("inf"), -float("inf")])
def test_a_query_that_is_not_finite(dev, mods, form, what):
    """Its own row becomes NaN, in whichever element it stands; every other row keeps its bits."""
    B, dec, ops = mods
    r = _rng(14000)
    heads, n, dim = 4, 2, 96
    M, pos0 = {"token": (1, 700), "rows": (3, 900), "tiles": (40, 300), "prefix in tiles": (7, 1000)}[form]
    table = _table(dim, pos0 + M + 1)
    q, k, v = _rows(r, M, heads * dim), _rows(r, M, n * dim), _rows(r, M, n * dim)
    cache, _ = _filled(dec, dev, r, n, dim, pos0 + M + 1, [pos0], table)

    def out(q):
        if form in ("rows", "tiles"):
            return dec.attn_prefill8(_t(q, dev), _t(k, dev), _t(v, dev), cache, _t(table, dev), pos0)
        if form == "token":
            return dec.Attention8(heads, cache, _t(q, dev), _t(k, dev), _t(v, dev), _t(np.array([pos0], np.int32), dev), _t(table, dev)).launch()
        own = dec.KvCache8(n, dim, 1, dev, sequences=M)
        return dec.Attention8(heads, own, _t(q, dev), _t(k, dev), _t(v, dev), _t(np.full(M, pos0, np.int32), dev), _t(table, dev), prefix=cache, prefix_len=pos0).launch()
    clean = out(q).cpu().reshape(M, heads, dim)
    assert bool(torch.isfinite(clean).all())
    for m, h, e in ((0, 1, 0), (M - 1, 3, dim - 1), (M // 2, 0, dim // 2 + 3)):
        bad = q.copy()
        bad[m, h * dim + e] = what
        got = out(bad).cpu().reshape(M, heads, dim)
        assert bool(torch.isnan(got[m, h]).all())
        got[m, h] = clean[m, h]
        assert torch.equal(got, clean)


def test_offsets_beyond_32_bits(dev, mods):
    """Sequences of a million positions, the last one's rows more than 2^32 bytes behind the first one's: writes at both ends, reads, a token's
    attention and a prompt's."""
    B, dec, ops = mods
    r = _rng(15000)
    heads, n, dim, most, seqs = 4, 4, 128, 1000000, 10
    assert (seqs - 1) * n * most * dim > 2 ** 32
    cache = dec.KvCache8(n, dim, most, dev, sequences=seqs)
    k, v = _rows(r, 70, n * dim), _rows(r, 70, n * dim)
    cache.write(_t(k, dev), _t(v, dev), most - 70, sequence=seqs - 1)
    for got, x in zip(cache.read(most - 70, 70, sequence=seqs - 1), (k, v)):
        codes, scale = _codes(x, dim)
        np.testing.assert_array_equal(got.cpu().numpy().reshape(70, n, dim), codes.astype(np.float32) * scale[..., None])
    assert not bool(cache.read(most - 140, 70, sequence=seqs - 1)[0].any()) and not bool(cache.read(most - 70, 70, sequence=seqs - 2)[0].any())
    small, table = dec.KvCache8(n, dim, 200, dev), _table(dim, 200)
    grown = torch.zeros((most, dim // 2, 2), device=dev)
    grown[:200] = _t(table, dev)
    q, k, v = (_t(_rows(r, 150, n * dim), dev) for _ in range(3))
    a = dec.attn_prefill8(q, k, v, cache, grown, 0, sequence=seqs - 1)
    b = dec.attn_prefill8(q, k, v, small, _t(table, dev), 0)
    assert torch.equal(a, b)                                    # (a prompt's plan does not depend on the cache's size)
    tokens = [_t(_rows(r, seqs, n * dim), dev) for _ in range(3)]
    pos = torch.full((seqs,), -1, dtype=torch.int32, device=dev)
    pos[-1] = 150
    out = dec.Attention8(heads, cache, *tokens, pos, grown).launch()[-1]
    one = dec.Attention8(heads, small, *(t[-1:].contiguous() for t in tokens), pos[-1:].contiguous(), _t(table, dev)).launch()[0]
    for x, y in zip(cache.read(0, 151, sequence=seqs - 1), small.read(0, 151)):
        assert torch.equal(x, y)
    # two orders of one sum, each within eight times the other tests' mean distance from the exact one
    assert float((out - one).abs().max()) <= 2 * 2.6e-6 * 8 * float(small.read(0, 151)[1].abs().max())


@pytest.mark.parametrize("heads,n,dim,pos0,M", [(3, 3, 64, 0, 300), (10, 5, 36, 20, 500), (28, 4, 128, 0, 130), (16, 2, 256, 5, 75), (12, 12, 64, 0, 900), (21, 7, 64, 0, 1500), (4, 1, 64, 100, 700)])
def test_prompts_of_few_key_heads(dev, mods, heads, n, dim, pos0, M):
    """Numbers of key heads that are no multiple of the dies: a head's blocks by strips, and what is left over at their ends."""
    _check_prompt(mods, dev, heads, n, dim, pos0, M, 64000 + pos0 + M, sample=sorted({0, 1, 31, 32, 33, M // 3, M // 2, M - 34, M - 2, M - 1}))
