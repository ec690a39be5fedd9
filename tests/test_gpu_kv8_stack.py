"""The 8-bit cache in use: DecoderStack(cache="int8") token by token and as a prompt, forks of it, streams and graphs."""
import numpy as np
import pytest

import oracle
import test_gpu_decoder as T
from oracle import decoder as D
from test_gpu_kv8 import _codes, _rows, _table

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
dev, mods = T.dev, T.mods


def _step8(h, pos, l, k_cache, v_cache, n_heads):
    """The oracle's layer step with the 8-bit cache: keys rotated and quantized as cached, values quantized."""
    d = h.shape[0] // n_heads
    y = D.rmsnorm(h, l["g_in"], 1e-5)
    q, k, v = (D.bitlinear_f32(y, l[n], l["s_" + n]) for n in "qkv")
    for cache, x in ((k_cache, D.rope(k, pos, n_heads).astype(np.float32)), (v_cache, np.asarray(v, np.float32))):
        codes, scale = _codes(x[None], d)
        cache[pos] = (codes[0] * scale[0][:, None].astype(np.float64)).reshape(-1)
    a = D.attention_decode(D.rope(q, pos, n_heads), k_cache[:pos + 1], v_cache[:pos + 1], n_heads)
    h = h + D.bitlinear_f32(D.rmsnorm(a, l["g_attn"], 1e-5), l["o"], l["s_o"])
    y = D.rmsnorm(h, l["g_post"], 1e-5)
    f = D.rmsnorm(D.gated_ffn_input(D.bitlinear_f32(y, l["gate"], l["s_gate"]), D.bitlinear_f32(y, l["up"], l["s_up"])), l["g_ffn"], 1e-5)
    return h + D.bitlinear_f32(f, l["down"], l["s_down"])


@pytest.mark.parametrize("hidden,ffn,n_heads,use_graph,fold", [(768, 1024, 12, False, True), (1536, 2048, 16, True, True), (200, 328, 5, True, False),
                                                               (768, 1024, 12, True, "gated")])
def test_token_loop_against_oracle(dev, mods, hidden, ffn, n_heads, use_graph, fold):
    """Bound and reason as in the bf16 stack's test of this name: a code that falls the other way in a quantizer moves everything behind it."""
    B, dec, ops = mods
    layers, g_final = T._make_layers(71000 + hidden, hidden, ffn, 2)
    gated, fold = fold == "gated", bool(fold)
    make = lambda: dec.DecoderStack(T._to_device(layers, dev, dec, ops, gated), T._t(g_final, dev), n_heads, 8, dev, fold_norm=fold, cache="int8")  # noqa: E731
    stack, eager = make(), make()
    if use_graph:
        stack.capture()
    r = T._rng(72000 + hidden)
    kcs, vcs = ([np.zeros((8, hidden)) for _ in layers] for _ in range(2))
    for pos in range(5):
        x = r.standard_normal((1, hidden)).astype(np.float32)
        for s in (stack, eager):
            s.h.copy_(T._t(x, dev))
        y, y2 = stack.step(), eager.step()
        assert torch.equal(y, y2)
        for a, b in zip(stack.layers, eager.layers):
            for n in ("k_codes", "v_codes", "k_scale", "v_scale"):
                assert torch.equal(getattr(a.attn.cache, n), getattr(b.attn.cache, n))
        h = x[0].astype(np.float64)
        for i, l in enumerate(layers):
            h = _step8(h, pos, l, kcs[i], vcs[i], n_heads)
        want, got = D.rmsnorm(h, g_final, 1e-5), y.cpu().numpy()[0].astype(np.float64)
        assert np.linalg.norm(got - want) <= 5e-2 * np.linalg.norm(want)


def test_prompt_then_tokens(dev, mods):
    """A prompt in two pieces and tokens behind it follow the same tokens taken one at a time: the first layer's cache is the same bits."""
    B, dec, ops = mods
    hidden, ffn, n_heads, max_pos = 256, 512, 4, 160
    layers, g_final = T._make_layers(73000, hidden, ffn, 2)
    a, b = (dec.DecoderStack(T._to_device(layers, dev, dec, ops), T._t(g_final, dev), n_heads, max_pos, dev, fold_norm=False, cache="int8") for _ in range(2))
    x = torch.randn((103, hidden), device=dev, generator=torch.Generator(device=dev).manual_seed(9))
    ya, yb = torch.cat([a.prefill(x[:70].contiguous()), a.prefill(x[70:100].contiguous())]), []
    for t in range(103):
        b.h.copy_(x[t:t + 1])
        yb.append(b.step().clone())
        if t >= 100:
            a.h.copy_(x[t:t + 1])
            ya = torch.cat([ya, a.step()])
    yb = torch.cat(yb)
    for n in ("k_codes", "v_codes", "k_scale", "v_scale"):
        assert torch.equal(getattr(a.layers[0].attn.cache, n), getattr(b.layers[0].attn.cache, n))
    assert float(torch.linalg.norm(ya - yb)) <= 5e-2 * float(torch.linalg.norm(yb))


@pytest.mark.parametrize("n,P,use_graph", [(1, 40, False), (3, 100, True), (3, 0, False), (9, 70, True)])
def test_fork_follows_its_sequences_one_by_one(dev, mods, n, P, use_graph):
    """n sequences behind a prompt, against n stacks that go on alone: the first layer's rows are the same bits, the hidden states within the
    bound of the token loop.  (Products of up to eight rows and of more.)"""
    B, dec, ops = mods
    hidden, ffn, n_heads, steps = 256, 512, 4, 6
    layers, g_final = T._make_layers(74000, hidden, ffn, 2)
    make = lambda: dec.DecoderStack(T._to_device(layers, dev, dec, ops), T._t(g_final, dev), n_heads, P + steps, dev, fold_norm=False, cache="int8")  # noqa: E731
    g = torch.Generator(device=dev).manual_seed(11)
    prompt, x = torch.randn((P, hidden), device=dev, generator=g), torch.randn((steps, n, hidden), device=dev, generator=g)
    stack = make()
    if P:
        stack.prefill(prompt)
    fork = stack.fork(n, steps)
    if use_graph:
        fork.capture()
    ys = []
    for t in range(steps):
        fork.h.copy_(x[t])
        ys.append(fork.step().clone())
    assert fork.pos.tolist() == [P + steps] * n
    with pytest.raises(RuntimeError):
        fork.step()
    for b in range(n):
        alone = make()
        if P:
            alone.prefill(prompt)
        for t in range(steps):
            alone.h.copy_(x[t, b:b + 1])
            y = alone.step()[0]
            assert float((ys[t][b] - y).norm()) <= 5e-2 * float(y.norm())
        mine, theirs = fork.layers[0][2].cache.read(0, steps, sequence=b), alone.layers[0].attn.cache.read(P, steps)
        assert torch.equal(mine[0], theirs[0]) and torch.equal(mine[1], theirs[1])


def test_a_stopped_sequence_is_left_alone(dev, mods):
    B, dec, ops = mods
    hidden, n_heads = 256, 4
    layers, g_final = T._make_layers(75000, hidden, 512, 1)
    stack = dec.DecoderStack(T._to_device(layers, dev, dec, ops), T._t(g_final, dev), n_heads, 64, dev, cache="int8", fold_norm=False)
    x = torch.randn((30, hidden), device=dev, generator=torch.Generator(device=dev).manual_seed(3))
    stack.prefill(x[:20].contiguous())
    a, b = stack.fork(3, 5), stack.fork(3, 5)
    a.capture()
    for t in range(4):
        if t == 2:
            a.stop(1)
            before = [c.clone() for c in (a.layers[0][2].cache.k_codes[1], a.layers[0][2].cache.v_scale[1])]
        for f in (a, b):
            f.h.copy_(x[20 + t:23 + t])
        ya, yb = a.step(), b.step()
        assert torch.equal(ya[0], yb[0]) and torch.equal(ya[2], yb[2])
    assert a.pos.tolist() == [24, -1, 24]
    assert torch.equal(before[0], a.layers[0][2].cache.k_codes[1]) and torch.equal(before[1], a.layers[0][2].cache.v_scale[1])


def test_refusals(dev, mods):
    B, dec, ops = mods
    layers, g_final = T._make_layers(76000, 128, 128, 1)
    make = lambda **kw: dec.DecoderStack(T._to_device(layers, dev, dec, ops), T._t(g_final, dev), 2, 8, dev, **kw)  # noqa: E731
    with pytest.raises(ValueError):
        make(cache="fp8")
    with pytest.raises(ValueError):
        make().fork(2, 4)
    with pytest.raises(ValueError):
        make(cache="int8").fork(0, 4)
    with pytest.raises(B.BitLinearError):
        dec.KvCache8(2, 62, 10, dev)
    with pytest.raises(B.BitLinearError):
        dec.KvCache8(2, 64, 10, dev, sequences=0)
    cache = dec.KvCache8(2, 64, 10, dev)
    k = torch.zeros((4, 128), device=dev)
    for args in ((k, k, 7), (k, k, -1)):
        with pytest.raises(B.BitLinearError):
            cache.write(*args)
    with pytest.raises(B.BitLinearError):
        cache.write(k, k, 0, sequence=1)
    with pytest.raises(B.BitLinearError):
        cache.read(5, 6)
    with pytest.raises(B.BitLinearError):
        cache.read(0, 0)
    with pytest.raises(TypeError):
        cache.write(k.half(), k.half(), 0)
    for bad in (lambda: cache.write(k, k[:3], 0), lambda: cache.write(k.t().contiguous().t(), k, 0), lambda: cache.write(k.cpu(), k, 0),
                lambda: cache.write(k, k, 0, torch.zeros((3, 32, 2), device=dev))):
        with pytest.raises(AssertionError):
            bad()
    pos, table = torch.zeros(1, dtype=torch.int32, device=dev), torch.zeros((10, 32, 2), device=dev)
    with pytest.raises(B.BitLinearError):
        dec.Attention8(3, cache, k[:1, :].repeat(1, 2)[:, :192].contiguous(), k[:1], k[:1], pos, table)    # three query heads on two key heads
    with pytest.raises(AssertionError):
        dec.Attention8(2, cache, k[:1], k[:1], k[:1], pos, table[:9])                                       # a table shorter than the cache
    with pytest.raises(AssertionError):
        dec.attn_prefill8(k, k, k, cache, table, 7)                                                         # ... or than the prompt's end


# ------------------------------------------------------------------------------------------------ streams and graphs

def _batch(dec, dev, seed, heads, n, dim, P, lengths):
    r = T._rng(seed)
    own, seqs = max(lengths) + 4, len(lengths)
    table = T._t(_table(dim, P + own), dev)
    cache, prefix = dec.KvCache8(n, dim, own, dev, sequences=seqs), dec.KvCache8(n, dim, max(1, P), dev)
    if P:
        prefix.write(T._t(_rows(r, P, n * dim), dev), T._t(_rows(r, P, n * dim), dev), 0, table)
    for b, m in enumerate(lengths):
        if m:
            cache.write(T._t(_rows(r, m, n * dim), dev), T._t(_rows(r, m, n * dim), dev), 0, table[P:].contiguous(), sequence=b)
    q, k, v = (T._t(_rows(r, seqs, w * dim), dev) for w in (heads, n, n))
    pos = T._t(np.array([P + m for m in lengths], np.int32), dev)
    return dec.Attention8(heads, cache, q, k, v, pos, table, prefix=prefix if P else None, prefix_len=P)


CASES = [(4, 4, 128, 0, [0]), (4, 4, 64, 0, [3000]), (4, 2, 96, 2000, [5, 300, 70]), (4, 1, 64, 700, [90] * 9), (32, 32, 64, 100, [9] * 20)]


@pytest.mark.parametrize("case", CASES)
def test_graph_replays_equal_eager_calls(dev, mods, case):
    """Captured, replayed with eager work and synchronizations in between, positions moving on the device: bit for bit the eager calls;
    a call repeated gives the same bits."""
    B, dec, ops = mods
    a, b = (_batch(dec, dev, 81000, *case) for _ in range(2))
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(s):
        with torch.cuda.graph(graph, stream=s):
            a.launch()          # (the first use of the kernel may be this one)
    torch.cuda.current_stream().wait_stream(s)
    for t in range(4):
        graph.replay()
        want = b.launch().clone()
        again = b.launch()
        torch.cuda.synchronize()
        assert torch.equal(want, again) and torch.equal(a.out, want)
        for n in ("k_codes", "v_codes", "k_scale", "v_scale"):
            assert torch.equal(getattr(a.cache, n), getattr(b.cache, n))
        for x in (a, b):
            pos = x._keep[3]
            pos.add_(1 if t < 3 else 0)
        (torch.randn(1000, 1000, device=dev) @ torch.randn(1000, 1000, device=dev)).sum().item()


def test_calls_on_other_streams(dev, mods):
    """Two prepared calls, each on a stream of its own at the same time, with their own scratch memory; write, prompt and read on a side stream."""
    B, dec, ops = mods
    calls = [_batch(dec, dev, 82000 + i, *c) for i, c in enumerate(CASES[1:4])]
    want = [c.launch().clone() for c in calls]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        for c in calls:
            c.out.fill_(-5.0)
        torch.cuda.synchronize()
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                c.launch()
        torch.cuda.synchronize()
        for w, c in zip(want, calls):
            assert torch.equal(w, c.out)
    r = T._rng(83000)
    n, dim, M = 2, 128, 150
    q, k, v = (T._t(_rows(r, M, n * dim), dev) for _ in range(3))
    table = T._t(_table(dim, 400), dev)
    got = []
    for s in (torch.cuda.current_stream(), torch.cuda.Stream()):
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            cache = dec.KvCache8(n, dim, 400, dev)
            cache.write(k, v, 0, table)
            out = dec.attn_prefill8(q, k, v, cache, table, M)
            got.append((out, *cache.read(0, 2 * M)))
        torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_a_captured_prompt(dev, mods):
    """attn_prefill8 under capture, replayed: split walks with their merging launch, several tiles per workgroup, and rows that meet by counters."""
    B, dec, ops = mods
    for heads, n, dim, pos0, M in ((4, 4, 64, 2000, 40), (2, 2, 128, 3000, 2), (32, 32, 64, 0, 1030)):
        r = T._rng(84000 + M)
        table = T._t(_table(dim, pos0 + M), dev)
        q, k, v = T._t(_rows(r, M, heads * dim), dev), T._t(_rows(r, M, n * dim), dev), T._t(_rows(r, M, n * dim), dev)
        cache = dec.KvCache8(n, dim, pos0 + M, dev)
        if pos0:
            cache.write(T._t(_rows(r, pos0, n * dim), dev), T._t(_rows(r, pos0, n * dim), dev), 0, table)
        want = dec.attn_prefill8(q, k, v, cache, table, pos0)
        out = torch.empty_like(want)
        s = torch.cuda.Stream()
        s.wait_stream(torch.cuda.current_stream())
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.stream(s):
            with torch.cuda.graph(graph, stream=s):
                dec.attn_prefill8(q, k, v, cache, table, pos0, out=out)
        torch.cuda.current_stream().wait_stream(s)
        for _ in range(4):
            out.fill_(3.0)
            graph.replay()
            torch.cuda.synchronize()
            assert torch.equal(out, want)
            torch.randn(500, 500, device=dev).sum().item()


def test_native_calls_are_the_ctypes_ones(dev, mods, monkeypatch):
    """write, read and attn_prefill8 in native code beside the Python path that they stand in for: the same bits, and for what they do not
    take as it is the same result or the same refusal."""
    B, dec, ops = mods
    assert B.calls()
    r = T._rng(85000)
    n, dim, M = 2, 96, 40
    wide = T._t(_rows(r, M, 2 * n * dim), dev)
    k, v, q = (T._t(_rows(r, M, w * n * dim), dev) for w in (1, 1, 3))
    table = T._t(_table(dim, 100), dev)
    half = wide.half()

    def outcomes():
        cache = dec.KvCache8(n, dim, 90, dev, sequences=2)
        calls = [
            lambda: cache.write(k, v, 3, table), lambda: cache.write(k.bfloat16(), v.bfloat16(), 50, sequence=1),
            lambda: cache.write(wide[:, :n * dim], wide[:, n * dim:], 47, table), lambda: cache.write(k[:1], v[:1], 89, table),
            lambda: cache.write(k, v, 51, table), lambda: cache.write(k, v, 0, table[:39]), lambda: cache.write(half[:, :n * dim], half[:, n * dim:], 0),
            lambda: cache.write(k, v, 0, table, 2), lambda: cache.write(k, v[:, :96], 0), lambda: cache.write(k[:0], v[:0], 0), lambda: cache.write(k, v.cpu(), 0),
            lambda: cache.write(k, v.bfloat16(), 0),
            lambda: cache.read(0, 90), lambda: cache.read(33, 50, torch.bfloat16, 1), lambda: cache.read(0, 91), lambda: cache.read(-1, 2), lambda: cache.read(0, 2, sequence=2),
            lambda: cache.read(0, 10 ** 9), lambda: cache.read(0, 4, torch.float16),
            lambda: dec.attn_prefill8(q, k, v, cache, table, 20), lambda: dec.attn_prefill8(q, k, v, cache, table, 50, 1, torch.zeros_like(q)),
            lambda: dec.attn_prefill8(q, k, v, cache, table, 51), lambda: dec.attn_prefill8(q[:, :96].contiguous(), k, v, cache, table, 0),
            lambda: dec.attn_prefill8(q[:, :100].contiguous(), k, v, cache, table, 0), lambda: dec.attn_prefill8(q, k[:39], v[:39], cache, table, 0),
            lambda: dec.attn_prefill8(q, k, v, cache, table[:59], 20), lambda: dec.attn_prefill8(q, k, v, cache, table, 0, 2),
            lambda: dec.attn_prefill8(q, k, v, cache, table, 0, 0, q[:39]), lambda: dec.attn_prefill8(q[:0], k[:0], v[:0], cache, table, 0)]
        got = []
        for call in calls:
            try:
                out = call()
                torch.cuda.synchronize()
                out = [t.clone() for t in (out if isinstance(out, tuple) else (out,)) if t is not None]
                got.append([t.cpu() for t in out + [cache.k_codes, cache.v_codes, cache.k_scale, cache.v_scale]])
            except Exception as e:      # noqa: BLE001 -- the kind and the words are what is compared
                got.append((type(e).__name__, str(e)))
        return got

    native = outcomes()
    monkeypatch.setattr(B, "_calls", False)
    for i, (a, b) in enumerate(zip(native, outcomes(), strict=True)):
        assert type(a) is type(b), (i, a, b)
        assert a == b if isinstance(a, tuple) else all(x.dtype == y.dtype and torch.equal(x, y) for x, y in zip(a, b, strict=True)), i
    refused = [isinstance(a, tuple) for a in native]
    assert refused == [False] * 4 + [True] * 8 + [False] * 2 + [True] * 5 + [False] * 2 + [True] * 8     # (one query head does not share out over two key heads)
