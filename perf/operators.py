"""The 8-bit key/value cache and the attention over it: what is timed, in plain form and as the framework's calls.

A layer's cache holds, for every position and key head, `dim` int8 codes and one fp32 scale, of the key and of the value. The
operators: rows written into the cache (rotated, quantized) and read back; one token's attention; the attention of several
sequences that share a prefix; a prompt's attention. Rotation and quantizer are fp32 operations, each rounded on its own.

Both forms work on the same buffers (per sequence and key head; S = dim rounded up to 16; positions in chunks of 64):
  k_codes  [chunk][block of up to 64 dims][row][dims]   row of position p: 16 (p % 4) + p % 64 // 4
  v_codes  [chunk][S][64]                               dim by dim, the chunk's positions side by side
  k_scale, v_scale  [positions]
"""
import math

import torch

own = False

DEV = "cuda"
THETA = 10000.0

# (query heads, key heads, head size) of the framework's models (125M to 100B), and shared key heads and sizes that fill no sixteen
SHAPES = [(12, 12, 64), (16, 16, 96), (32, 32, 64), (32, 32, 48), (20, 20, 128), (32, 32, 120), (32, 32, 128), (40, 40, 128),
          (52, 52, 128), (64, 64, 128), (32, 8, 128), (64, 8, 128), (28, 4, 128), (12, 4, 100), (16, 2, 256), (10, 5, 36)]


def listed():
    return [
        # a short prompt's rows behind 27 others, a small model: nothing fills a chunk, latency
        dict(name="cache_37_small", kind="cache", heads=12, keys=12, dim=64, pos=27, M=37, dtype="float32"),
        # 2000 rows of a 7B model's bf16 projections into the cache and out again: the stream of a long prompt
        dict(name="cache_2000_7b", kind="cache", heads=32, keys=32, dim=128, pos=0, M=2000, dtype="bfloat16"),
        # the first words of an answer, a small model: the smallest call
        dict(name="token_17_small", kind="token", heads=12, keys=12, dim=64, pos=17),
        # a token deep in a conversation on the 7B shape
        dict(name="token_8k_7b", kind="token", heads=32, keys=32, dim=128, pos=8000),
        # a token behind a book, query heads in groups that share a key head
        dict(name="token_100k_grouped", kind="token", heads=64, keys=8, dim=128, pos=100003),
        # three answers to one question, a head size that fills no 64
        dict(name="batch_3_700m", kind="batch", heads=16, keys=16, dim=96, prefix=517, B=3, own=129),
        # eight sequences behind a long shared prompt on the 7B shape
        dict(name="batch_8_7b", kind="batch", heads=32, keys=32, dim=128, prefix=8000, B=8, own=300),
        # a served batch: sequences behind a common system prompt, shared key heads
        dict(name="batch_32_grouped", kind="batch", heads=32, keys=8, dim=128, prefix=2500, B=32, own=1000),
        # five drafted tokens looked at together behind a long cache
        dict(name="prompt_5_8k", kind="prompt", heads=32, keys=32, dim=128, pos=8000, M=5),
        # a prompt that fills no tile, behind a cache that ends inside a chunk, head size 120
        dict(name="prompt_77_ragged", kind="prompt", heads=32, keys=32, dim=120, pos=1001, M=77),
        # a prompt's second piece on the 7B shape
        dict(name="prompt_512_7b", kind="prompt", heads=32, keys=32, dim=128, pos=512, M=512),
        # a long prompt at once: the largest contraction
        dict(name="prompt_2048_7b", kind="prompt", heads=32, keys=32, dim=128, pos=0, M=2048),
    ]


# ---- drawing ---------------------------------------------------------------------------------------------------------

def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    heads, keys, dim = rng.choice(SHAPES)
    kind = rng.choice(["cache", "token", "token", "batch", "batch", "batch", "prompt", "prompt", "prompt"])
    c = dict(kind=kind, heads=heads, keys=keys, dim=dim)
    if kind == "cache":
        return dict(c, pos=rng.choice([0, _log_int(rng, 1, 3000)]), M=_log_int(rng, 1, 2000 * 4096 // max(4096, keys * dim)),
                    dtype=rng.choice(["float32", "bfloat16"]))
    if kind == "token":
        return dict(c, pos=_log_int(rng, 1, 100003 * 1024 // max(1024, keys * dim)) - 1)
    if kind == "batch":
        while True:
            c.update(prefix=rng.choice([0, _log_int(rng, 1, 16000)]), B=_log_int(rng, 2, 64), own=_log_int(rng, 1, 2000))
            if (c["prefix"] + c["B"] * c["own"]) * keys * dim <= 25000 * 4096 and (c["prefix"] + c["own"]) * c["B"] * heads * dim <= 32 * 3500 * 4096:
                return c
    while True:
        c.update(pos=rng.choice([0, _log_int(rng, 1, 16000)]), M=_log_int(rng, 2, 2048))
        if c["M"] * (c["pos"] + c["M"] / 2) * heads * dim <= 2048 * 1024 * 4096:
            return c


# ---- inputs, from the seed alone ----------------------------------------------------------------------------------------

def _gen(seed, what):
    return torch.Generator(device=DEV).manual_seed(seed * 1009 + what)


def _normal(seed, what, *shape):
    return torch.randn(shape, device=DEV, generator=_gen(seed, what))


def _rows(seed, what, M, heads, dim):
    """Projections of M tokens: normal values, some channels of a head larger than others, tokens of different size."""
    channel = torch.exp(0.5 * _normal(seed, what + 500, heads, dim))
    token = torch.exp(0.3 * _normal(seed, what + 501, M, 1, 1))
    return (_normal(seed, what, M, heads, dim) * channel * token * 0.7).reshape(M, heads * dim)


def _table(dim, positions):
    """[positions, dim / 2, 2]: cosine and sine, angles in 64 bits, kept in 32."""
    i = torch.arange(dim // 2, device=DEV, dtype=torch.float64)
    a = torch.arange(positions, device=DEV, dtype=torch.float64)[:, None] * THETA ** (-2.0 * i / dim)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _chunks(case):
    return -(-_capacity(case) // 64)


def _capacity(case):
    """Positions of a sequence's own cache."""
    return {"cache": lambda: case["pos"] + case["M"], "token": lambda: case["pos"] + 1, "batch": lambda: case["own"] + 1,
            "prompt": lambda: case["pos"] + case["M"]}[case["kind"]]()


def _sides(case):
    """(sequences, positions filled already, first position's angle, chunks) of the caches of a case: the prefix first, then the own ones."""
    if case["kind"] == "batch":
        return [(1, case["prefix"], 0, -(-max(1, case["prefix"]) // 64)), (case["B"], case["own"], case["prefix"], _chunks(case))]
    return [(1, case["pos"], 0, _chunks(case))]


def _own_lengths(case, seed):
    """Rows that each sequence of a batch has behind the prefix before this step."""
    return torch.randint(0, case["own"] + 1, (case["B"],), dtype=torch.int32, device=DEV, generator=_gen(seed, 7))


def _filled(case, seed, table):
    """The caches' buffers with the rows of the positions before this call."""
    keys, dim = case["keys"], case["dim"]
    size = -(-dim // 16) * 16
    caches = []
    for i, (sequences, rows, first, chunks) in enumerate(_sides(case)):
        cache = {n: torch.zeros((sequences, keys, chunks * 64 * size), dtype=torch.int8, device=DEV) for n in ("k_codes", "v_codes")}
        cache |= {n: torch.zeros((sequences, keys, chunks * 64), device=DEV) for n in ("k_scale", "v_scale")}
        for b in range(sequences if rows else 0):
            for r in range(0, rows, 16384):       # (a long cache a piece at a time)
                n = min(16384, rows - r)
                at = torch.arange(r, r + n, device=DEV)
                what = 1000 * (i + 1) + 10 * (b * 64 + r // 16384)
                _store(cache, b, at, _rotate(_rows(seed, what, n, keys, dim), table[first + r:first + r + n]), _rows(seed, what + 1, n, keys, dim), keys)
        caches.append(cache)
    return caches


def prepare(case, seed):
    kind, heads, keys, dim = case["kind"], case["heads"], case["keys"], case["dim"]
    M = case.get("B", case.get("M", 1))
    first = case.get("prefix", 0)
    table = _table(dim, first + _capacity(case))
    st = dict(kind=kind, heads=heads, keys=keys, dim=dim, table=table, caches=_filled(case, seed, table), first=first)
    st["q"], st["k"], st["v"] = _rows(seed, 1, M, heads, dim), _rows(seed, 2, M, keys, dim), _rows(seed, 3, M, keys, dim)
    if kind == "cache":
        st["k"], st["v"] = (st[n].to(getattr(torch, case["dtype"])) for n in "kv")
    if kind in ("cache", "prompt"):
        st["pos"], st["M"] = case["pos"], M
    else:
        st["pos"] = torch.full((1,), case["pos"], dtype=torch.int32, device=DEV) if kind == "token" else case["prefix"] + _own_lengths(case, seed)
        st["shared"] = case.get("prefix", 0)
    if own:
        _handles(st, case)
    return st


def _handles(st, case):
    """The framework's caches around the same rows, and the prepared launch of a token loop."""
    from paper_2410_16144_amd import decoder
    made = []
    positions = [case["prefix"], _capacity(case)] if case["kind"] == "batch" else [_capacity(case)]
    for cache, n in zip(st["caches"], positions):
        made.append(decoder.KvCache8(case["keys"], case["dim"], max(1, n), torch.device(DEV), sequences=cache["k_codes"].shape[0]))
        for name in cache:
            getattr(made[-1], name).copy_(cache[name])
            cache[name] = getattr(made[-1], name)
    st["cache"] = made[-1]
    if case["kind"] in ("token", "batch"):
        prefix = made[0] if case.get("prefix", 0) else None
        st["attention"] = decoder.Attention8(st["heads"], made[-1], st["q"], st["k"], st["v"], st["pos"], st["table"], prefix=prefix, prefix_len=case.get("prefix", 0))


# ---- one pass -----------------------------------------------------------------------------------------------------------

def run(st):
    if own:
        from paper_2410_16144_amd import decoder
        if st["kind"] == "cache":
            st["cache"].write(st["k"], st["v"], st["pos"], st["table"])
            k, v = st["cache"].read(st["pos"], st["M"], dtype=st["k"].dtype)
            return {"k": k, "v": v, **st["caches"][-1]}
        if st["kind"] == "prompt":
            out = decoder.attn_prefill8(st["q"], st["k"], st["v"], st["cache"], st["table"], st["pos"])
        else:
            out = st["attention"].launch()
        return {"out": out, **st["caches"][-1]}
    return {"cache": _plain_cache, "token": _plain_batch, "batch": _plain_batch, "prompt": _plain_prompt}[st["kind"]](st)


def _rotate(x, table):
    """x [rows, heads * dim]; table [rows, dim / 2, 2]. Pairs (i, i + dim / 2) of a head."""
    rows, half = x.shape[0], table.shape[1]
    x = x.float().view(rows, -1, 2, half)
    c, s = table[:, None, :, 0], table[:, None, :, 1]
    return torch.stack([x[:, :, 0] * c - x[:, :, 1] * s, x[:, :, 0] * s + x[:, :, 1] * c], 2).reshape(rows, -1)


def _quantize(x, heads):
    """Codes [rows, heads, dim] and scales [rows, heads] of fp32 rows."""
    x = x.view(x.shape[0], heads, -1)
    amax = x.abs().amax(-1)
    most = torch.full_like(amax, 127.0)
    inv = most / amax                         # (a quotient of two tensors: torch multiplies by the reciprocal of a number)
    dead = ~torch.isfinite(inv)
    codes = torch.where(dead[..., None], 0.0, (x * inv[..., None]).round().clamp(-128, 127))
    return codes.to(torch.int8), torch.where(dead, 0.0, amax / most)


def _places(at, dim):
    """Where the codes of positions `at` lie in a head's buffers: [rows, dim] offsets of keys and of values."""
    size = -(-dim // 16) * 16
    e = torch.arange(dim, device=DEV)
    chunk, p = (at // 64)[:, None] * (64 * size), (at % 64)[:, None]
    block = e // 64
    width = (size - 64 * block).clamp(max=64)
    return chunk + block * 4096 + (16 * (p % 4) + p // 4) * width + e % 64, chunk + e * 64 + p


def _store(cache, sequence, at, k, v, keys):
    """Rows k, v (fp32, keys rotated) into positions `at`; sequence: a number, or one for each row."""
    dim = k.shape[1] // keys
    places = _places(at, dim)
    head = torch.arange(keys, device=DEV)
    seq = sequence if isinstance(sequence, int) else sequence[:, None, None]
    for name, x, place in (("k", k, places[0]), ("v", v, places[1])):
        codes, scale = _quantize(x, keys)
        cache[name + "_codes"][seq, head[None, :, None], place[:, None, :]] = codes
        cache[name + "_scale"][seq if isinstance(seq, int) else seq[..., 0], head[None, :], at[:, None]] = scale


def _values(cache, dim):
    """What a cache stands for: keys and values [sequences, heads, positions, dim] in fp32."""
    n, h, bytes_ = cache["k_codes"].shape
    size = -(-dim // 16) * 16
    chunks = bytes_ // (64 * size)
    k = cache["k_codes"].view(n, h, chunks, 64 * size)
    blocks = [k[..., 64 * e:64 * min(e + 64, size)].reshape(n, h, chunks, 4, 16, -1).transpose(3, 4).reshape(n, h, chunks * 64, -1) for e in range(0, size, 64)]
    k = torch.cat(blocks, -1)[..., :dim].float() * cache["k_scale"][..., None]
    v = cache["v_codes"].view(n, h, chunks, size, 64).transpose(3, 4).reshape(n, h, chunks * 64, size)[..., :dim].float() * cache["v_scale"][..., None]
    return k, v


def _plain_cache(st):
    cache, at = st["caches"][-1], torch.arange(st["pos"], st["pos"] + st["M"], device=DEV)
    rows = st["table"][st["pos"]:st["pos"] + st["M"]]
    _store(cache, 0, at, _rotate(st["k"], rows), st["v"].float(), st["keys"])
    head, got = torch.arange(st["keys"], device=DEV)[:, None], []
    for name, place in zip("kv", _places(at, st["dim"])):
        x = cache[name + "_codes"][0][head[None], place[:, None]].float() * cache[name + "_scale"][0][:, at].t()[..., None]
        got.append(x.reshape(st["M"], -1).to(st["k"].dtype))
    return {"k": got[0], "v": got[1], **cache}


def _plain_batch(st):
    """One token of each sequence, behind the prefix and its own rows."""
    cache, heads, keys, dim = st["caches"][-1], st["heads"], st["keys"], st["dim"]
    pos = st["pos"].long()
    B, at, rows = pos.shape[0], pos - st["first"], st["table"][pos]
    _store(cache, torch.arange(B, device=DEV), at, _rotate(st["k"], rows), st["v"], keys)
    q = _rotate(st["q"], rows).view(B, keys, heads // keys, dim) / math.sqrt(dim)
    k, v = _values(cache, dim)
    beyond = torch.arange(k.shape[2], device=DEV) > at[:, None]
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).masked_fill(beyond[:, None, None], -math.inf)
    if not st["shared"]:
        out = torch.matmul(torch.softmax(s, -1), v)
    else:
        n = st["shared"]
        pk, pv = (x[0, :, :n] for x in _values(st["caches"][0], dim))
        qs = q.permute(1, 0, 2, 3).reshape(keys, -1, dim)                     # a key head's rows of all sequences
        ps = torch.matmul(qs, pk.transpose(1, 2).contiguous()).view(keys, B, -1, n).permute(1, 0, 2, 3)
        w = torch.softmax(torch.cat([ps, s], -1), -1)
        out = torch.matmul(w[..., :n].permute(1, 0, 2, 3).reshape(keys, -1, n), pv.contiguous()).view(keys, B, -1, dim).permute(1, 0, 2, 3)
        out = out + torch.matmul(w[..., n:].contiguous(), v)
    return {"out": out.reshape(B, heads * dim), **cache}


def _plain_prompt(st):
    cache, heads, keys, dim, M = st["caches"][-1], st["heads"], st["keys"], st["dim"], st["M"]
    at = torch.arange(st["pos"], st["pos"] + M, device=DEV)
    rows = st["table"][st["pos"]:st["pos"] + M]
    _store(cache, 0, at, _rotate(st["k"], rows), st["v"], keys)
    q = _rotate(st["q"], rows).view(M, keys, heads // keys, dim).permute(1, 2, 0, 3).reshape(keys, -1, dim) / math.sqrt(dim)
    k, v = (x[0, :, :st["pos"] + M] for x in _values(cache, dim))
    s = torch.matmul(q, k.transpose(1, 2).contiguous()).view(keys, heads // keys, M, -1)
    s = s.masked_fill(torch.arange(st["pos"] + M, device=DEV) > at[:, None], -math.inf)
    out = torch.matmul(torch.softmax(s, -1).view(keys, -1, st["pos"] + M), v.contiguous())
    return {"out": out.view(keys, heads // keys, M, dim).permute(2, 0, 1, 3).reshape(M, heads * dim), **cache}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------

def work(case):
    kind, n, heads, d = case["kind"], case["keys"] * case["dim"], case["heads"] * case["dim"], case["dim"]
    row = 2 * n + 8 * case["keys"]                                   # a position's codes and scales, key and value
    if kind == "cache":
        e = 4 if case["dtype"] == "float32" else 2
        return {"bytes": case["M"] * (4 * n * e + 2 * row + 4 * d), "flops": 10 * case["M"] * n}
    M = case.get("B", case.get("M", 1))
    inout = M * (8 * heads + 8 * n + 4 * d)
    if kind == "batch":                                              # (a sequence has half of `own` rows on average)
        mine = case["B"] * (case["own"] / 2 + 1)
        return {"bytes": inout + (case["prefix"] + mine) * row, "flops": 4 * heads * (case["B"] * case["prefix"] + mine)}
    return {"bytes": inout + (case["pos"] + M) * row, "flops": 4 * heads * (M * case["pos"] + M * (M + 1) / 2)}


# ---- the same in 64 bits ---------------------------------------------------------------------------------------------------

def _fp32(x):
    """One fp32 operation's rounding of a result that 64 bits hold."""
    return x.float().double()


def _exact_rows(k, v, table, keys, dim):
    """What rows stand for once they are in the cache: keys, values [rows, heads, dim] and their scales. The definition decides in fp32
    operations; each is done here in 64 bits and rounded."""
    half = dim // 2
    k = k.double().reshape(-1, keys, dim)
    c, s = table.double()[:, None, :, 0], table.double()[:, None, :, 1]
    a, b = k[..., :half], k[..., half:]
    k = torch.cat([_fp32(_fp32(a * c) - _fp32(b * s)), _fp32(_fp32(a * s) + _fp32(b * c))], -1)
    got = []
    for x in (k, v.double().reshape(-1, keys, dim)):
        largest = x.abs().max(-1, keepdim=True).values
        inv = _fp32(127.0 / largest)
        code = torch.round(_fp32(x * inv))
        scale = _fp32(largest / 127.0)
        alive = torch.isfinite(inv)
        got += [torch.where(alive, code * scale, 0.0), torch.where(alive, scale, 0.0)[..., 0]]
    return got


def _exact_past(case, seed, table):
    """Keys and values of the filled positions: for each cache, for each sequence, (keys, values, scales of both) [rows, heads, ...]."""
    keys, dim = case["keys"], case["dim"]
    caches = []
    for i, (sequences, rows, first, _) in enumerate(_sides(case)):
        cache = []
        for b in range(sequences):
            parts = []
            for r in range(0, rows, 16384):
                n, what = min(16384, rows - r), 1000 * (i + 1) + 10 * (b * 64 + r // 16384)
                parts.append(_exact_rows(_rows(seed, what, n, keys, dim), _rows(seed, what + 1, n, keys, dim), table[first + r:first + r + n], keys, dim))
            empty = [torch.zeros((0, keys, dim), device=DEV, dtype=torch.float64)] * 2 + [torch.zeros((0, keys), device=DEV, dtype=torch.float64)] * 2
            cache.append([torch.cat(x) for x in zip(*parts)] if parts else [empty[0], empty[2], empty[1], empty[3]])
        caches.append(cache)
    return caches


def _exact_attention(q, k, v, group, seen):
    """Queries [M, heads, dim] over keys, values [rows, key heads, dim]; query m sees the first seen[m] rows."""
    out = torch.empty_like(q)
    for h in range(q.shape[1]):
        s = q[:, h] @ k[:, h // group].t() / math.sqrt(q.shape[2])
        s[torch.arange(k.shape[0], device=DEV)[None] >= seen[:, None]] = -math.inf
        w = torch.exp(s - s.max(1, keepdim=True).values)
        out[:, h] = (w @ v[:, h // group]) / w.sum(1, keepdim=True)
    return out.reshape(q.shape[0], -1)


def _exact_scales(past, sequences, case, at, new):
    """A cache's buffer of scales: those of the rows before, the call's own at positions `at`, zero behind them."""
    full = torch.zeros((sequences, case["keys"], _chunks(case) * 64), device=DEV, dtype=torch.float64)
    for b, p in enumerate(past):
        full[b, :, :p.shape[0]] = p.t()
    for i, p in enumerate(at):
        full[i if sequences > 1 else 0, :, p] = new[i]
    return full


def exact(case, seed):
    kind, heads, keys, dim = case["kind"], case["heads"], case["keys"], case["dim"]
    M, first = case.get("B", case.get("M", 1)), case.get("prefix", 0)
    table = _table(dim, first + _capacity(case))
    q, k, v = _rows(seed, 1, M, heads, dim), _rows(seed, 2, M, keys, dim), _rows(seed, 3, M, keys, dim)
    if kind == "cache":
        k, v = (x.to(getattr(torch, case["dtype"])) for x in (k, v))
    past = _exact_past(case, seed, table)
    if kind == "batch":
        at = _own_lengths(case, seed).tolist()
    else:
        at = list(range(case["pos"], case["pos"] + M))
    angles = table[[first + p for p in at]]
    nk, nks, nv, nvs = _exact_rows(k, v, angles, keys, dim)
    sequences = M if kind == "batch" else 1
    buffers = {"k_codes": None, "v_codes": None}
    for name, i, new in (("k_scale", 1, nks), ("v_scale", 3, nvs)):
        buffers[name] = _exact_scales([s[i] for s in past[-1]], sequences, case, at, new)
    if kind == "cache":
        return {"k": nk.reshape(M, -1), "v": nv.reshape(M, -1), **buffers}
    qd, half = q.double().view(M, heads, dim), dim // 2
    c, s = angles.double()[:, None, :, 0], angles.double()[:, None, :, 1]
    qd = torch.cat([qd[..., :half] * c - qd[..., half:] * s, qd[..., :half] * s + qd[..., half:] * c], -1)
    if kind != "batch":
        kk, vv = torch.cat([past[0][0][0], nk]), torch.cat([past[0][0][2], nv])
        out = _exact_attention(qd, kk, vv, heads // keys, torch.tensor(at, device=DEV) + 1)
    else:
        out = torch.empty((M, heads * dim), device=DEV, dtype=torch.float64)
        for b in range(M):
            kk = torch.cat([past[0][0][0], past[1][b][0][:at[b]], nk[b:b + 1]])
            vv = torch.cat([past[0][0][2], past[1][b][2][:at[b]], nv[b:b + 1]])
            out[b] = _exact_attention(qd[b:b + 1], kk, vv, heads // keys, torch.tensor([kk.shape[0]], device=DEV))[0]
    return {"out": out, **buffers}
