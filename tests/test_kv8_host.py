"""The 8-bit cache without a GPU: refusals, sizes, structures as the header has them, the layout's arithmetic and the plan of the launches."""
import ctypes
import os
import subprocess

import pytest

from paper_2410_16144_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 0x10000   # an aligned address that nobody reads: validation comes first


def _st(f, *a):
    with pytest.raises(B.BitLinearError) as e:
        f(*a)
    return e.value.status


def _cache(**kw):
    f = dict(k_codes_dev=P, v_codes_dev=P, k_scale_dev=P, v_scale_dev=P, n_heads=4, head_dim=64, max_pos=100, sequences=2)
    return B.Kv8Cache(**dict(f, **kw))


def test_structures_as_the_header_has_them(tmp_path):
    names = {"bl_kv8_cache": B.Kv8Cache, "bl_kv8_write_args": B.Kv8WriteArgs, "bl_kv8_read_args": B.Kv8ReadArgs, "bl_attn8_args": B.Attn8Args,
             "bl_attn8_prefill_args": B.Attn8PrefillArgs}
    lines = "".join('printf("%%zu", sizeof(%s));' % n + "".join('printf(" %%zu", offsetof(%s, %s));' % (n, f[0]) for f in c._fields_) + 'printf("\\n");'
                    for n, c in names.items())
    src = tmp_path / "sizes.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "bitlinear_decoder.h"\nint main(void) {' + lines + "return 0;}")
    exe = str(tmp_path / "sizes")
    subprocess.check_call(["gcc", "-std=c11", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), str(src), "-o", exe])
    for line, (n, c) in zip(subprocess.check_output([exe], text=True).splitlines(), names.items()):
        assert [int(x) for x in line.split()] == [ctypes.sizeof(c)] + [getattr(c, f[0]).offset for f in c._fields_], n


def test_sizes_of_the_buffers():
    assert B.bl_kv8_code_bytes(32, 128, 8192) == 32 * 128 * 8192 and B.bl_kv8_scale_count(32, 8192) == 32 * 8192
    assert B.bl_kv8_code_bytes(3, 100, 65) == 3 * 112 * 128 and B.bl_kv8_scale_count(3, 65) == 3 * 128
    assert B.bl_kv8_code_bytes(1, 4, 1) == 16 * 64
    for bad in ((0, 64, 10), (4, 62, 10), (4, 260, 10), (4, 64, 0), (65536, 64, 10), (4, 64, 64 * 65535 + 1)):
        assert B.bl_kv8_code_bytes(*bad) == 0
    assert B.bl_kv8_scale_count(0, 10) == 0 and B.bl_kv8_scale_count(1, 0) == 0
    assert B.bl_kv8_code_bytes(65535, 256, 64 * 65535) == 65535 * 256 * 64 * 65535    # beyond 32 bits


def test_refusals_of_write_and_read():
    def write(cache=None, **kw):
        a = dict(k=P, v=P, table=P, ld=256, dt=B.BL_F32, sequence=0, pos0=10, M=5)
        a.update(kw)
        return _st(B.bl_kv8_write, cache or _cache(), *a.values())

    def read(cache=None, **kw):
        a = dict(k=P, v=P, ld=256, dt=B.BL_F32, sequence=0, pos0=10, M=5)
        a.update(kw)
        return _st(B.bl_kv8_read, cache or _cache(), *a.values())
    for f in (write, read):
        assert f(_cache(k_codes_dev=None)) == f(_cache(v_codes_dev=None)) == f(_cache(k_scale_dev=None)) == f(_cache(v_scale_dev=None)) == B.BL_ERR_NULL
        for kw in (dict(n_heads=0), dict(head_dim=62), dict(head_dim=0), dict(max_pos=0), dict(sequences=0), dict(n_heads=5)):
            assert f(_cache(**kw)) == B.BL_ERR_SHAPE, kw
        for kw in (dict(sequence=2), dict(sequence=-1), dict(pos0=-1), dict(pos0=96), dict(M=0), dict(M=-3), dict(M=91), dict(ld=255), dict(pos0=2147483647)):
            assert f(**kw) == B.BL_ERR_SHAPE, kw
        assert f(dt=2) == B.BL_ERR_DTYPE
        assert f(_cache(k_codes_dev=P + 8)) == f(_cache(v_codes_dev=P + 4)) == f(_cache(k_scale_dev=P + 4)) == f(_cache(v_scale_dev=P + 8)) == B.BL_ERR_ALIGN
        assert f(k=P + 2) == f(v=P + 2) == f(k=P + 1, dt=B.BL_BF16) == B.BL_ERR_ALIGN
    assert write(k=0) == write(v=0) == B.BL_ERR_NULL and read(k=0, v=0) == B.BL_ERR_NULL
    assert write(table=P + 4) == B.BL_ERR_ALIGN
    assert _st(B.bl_kv8_write, None, P, P, P, 256, 0, 0, 0, 1) == _st(B.bl_kv8_read, None, P, P, 256, 0, 0, 0, 1) == B.BL_ERR_NULL


def test_refusals_of_the_token_attention():
    def call(cache=None, n_q=8, prefix=None, prefix_len=0, **kw):
        a = dict(q=P, k=P, v=P, pos=P, table=P, out=P, scratch=P)
        a.update(kw)
        return _st(B.bl_attn8_decode, B.make_attn8_args(*a.values(), cache or _cache(), n_q, prefix, prefix_len))
    for name in ("q", "k", "v", "pos", "table", "out", "scratch"):
        assert call(**{name: 0}) == B.BL_ERR_NULL
    assert call(_cache(k_codes_dev=None)) == B.BL_ERR_NULL and call(prefix_len=3) == B.BL_ERR_NULL      # a prefix without buffers
    for n_q in (0, -4, 6, 4 * 65):
        assert call(n_q=n_q) == B.BL_ERR_SHAPE
    for kw in (dict(head_dim=6), dict(sequences=0), dict(sequences=B.BL_ATTN8_MAX_BATCH + 1), dict(max_pos=-1)):
        assert call(_cache(**kw)) == B.BL_ERR_SHAPE
    assert call(prefix_len=-1) == B.BL_ERR_SHAPE and call(prefix=_cache(), prefix_len=101) == B.BL_ERR_SHAPE
    assert call(prefix=_cache(n_heads=8), prefix_len=5) == call(prefix=_cache(head_dim=60), prefix_len=5) == B.BL_ERR_SHAPE
    for kw in ({}, dict(k_codes_dev=P + (1 << 30)), dict(k_codes_dev=P + 2048, v_codes_dev=P + (1 << 30)), dict(k_codes_dev=P - 4096, v_codes_dev=P + (1 << 30))):
        assert call(prefix=_cache(**kw), prefix_len=5) == B.BL_ERR_SHAPE      # a prefix in the memory of the sequences' own rows
    for name, off in (("q", 2), ("k", 2), ("v", 1), ("pos", 2), ("table", 4), ("out", 4), ("scratch", 8)):
        assert call(**{name: P + off}) == B.BL_ERR_ALIGN
    assert call(prefix=_cache(v_scale_dev=P + 4), prefix_len=5) == B.BL_ERR_ALIGN


def test_a_prefix_has_memory_of_its_own():
    """None of its codes and scales may lie in any of the sequences' buffers, of whatever kind: they are written while it is read."""
    own, far = _cache(k_codes_dev=1 << 32, v_codes_dev=2 << 32, k_scale_dev=3 << 32, v_scale_dev=4 << 32), [(i + 5) << 32 for i in range(4)]
    names = [f[0] for f in B.Kv8Cache._fields_[:4]]
    codes, scales = B.bl_kv8_code_bytes(4, 64, 100), 4 * B.bl_kv8_scale_count(4, 100)

    def call(prefix, q=P):
        return _st(B.bl_attn8_decode, B.make_attn8_args(q, P, P, P, P, P, P, own, 8, prefix, 5))
    assert call(_cache(**dict(zip(names, far))), q=P + 2) == B.BL_ERR_ALIGN          # (nothing wrong with this one)
    for i, name in enumerate(names):
        for j in range(4):
            mine, theirs = (scales if i >= 2 else codes), 2 * (scales if j >= 2 else codes)
            for at in (0, theirs - 16, 16 - mine):
                assert call(_cache(**dict(zip(names, far), **{name: ((j + 1) << 32) + at}))) == B.BL_ERR_SHAPE, (name, j, at)
            for at in (theirs, -mine):
                assert call(_cache(**dict(zip(names, far), **{name: ((j + 1) << 32) + at})), q=P + 2) == B.BL_ERR_ALIGN, (name, j, at)


def test_refusals_of_the_prompt_attention():
    def call(cache=None, n_q=8, sequence=0, pos0=10, M=20, **kw):
        a = dict(q=P, k=P, v=P, table=P, out=P, scratch=P)
        a.update(kw)
        return _st(B.bl_attn8_prefill, *a.values(), cache or _cache(), n_q, sequence, pos0, M)
    for name in ("q", "k", "v", "table", "out", "scratch"):
        assert call(**{name: 0}) == B.BL_ERR_NULL
    assert call(_cache(v_codes_dev=None)) == B.BL_ERR_NULL
    for kw in (dict(n_q=7), dict(n_q=0), dict(n_q=260), dict(sequence=2), dict(sequence=-1), dict(pos0=-1), dict(pos0=81), dict(M=0), dict(M=65536)):
        assert call(**kw) == B.BL_ERR_SHAPE, kw
    for name, off in (("q", 2), ("k", 2), ("v", 2), ("table", 4), ("out", 4), ("scratch", 8)):
        assert call(**{name: P + off}) == B.BL_ERR_ALIGN


def test_scratch_sizes():
    assert B.bl_attn8_scratch_bytes(32, 32, 128, 64, 1, 0) == 32 * 32 * 4                            # one workgroup per head
    for bad in ((31, 32, 128, 64, 1, 0), (32, 32, 130, 64, 1, 0), (32, 32, 128, 0, 1, 0), (32, 32, 128, 64, 0, 0), (32, 32, 128, 64, 1, -1)):
        assert B.bl_attn8_scratch_bytes(*bad) == 0
    assert B.bl_attn8_prefill_scratch_bytes(8, 4, 64, 0, 0) == B.bl_attn8_prefill_scratch_bytes(8, 3, 64, 0, 5) == 0
    assert B.bl_attn8_prefill_scratch_bytes(8, 4, 64, 0, 5) > 0


def test_batches_and_prompts_too_large_for_a_launch():
    """A launch has less than 2^32 threads: what needs more is refused ahead of every launch, a prompt's write included."""
    assert B.bl_attn8_scratch_bytes(65535, 65535, 4, 1, 64, 0) > 0 and B.bl_attn8_scratch_bytes(65535, 65535, 4, 1, 1024, 0) == 0
    assert B.bl_attn8_scratch_bytes(32000, 32000, 4, 1, 1024, 5) > 0 and B.bl_attn8_scratch_bytes(65535, 65535, 4, 1, 1024, 5) == 0
    assert B.bl_attn8_prefill_scratch_bytes(65535, 65535, 4, 0, 60000) > 0 and B.bl_attn8_prefill_scratch_bytes(65535, 65535, 4, 0, 65535) == 0
    far = dict(k_codes_dev=1 << 44, v_codes_dev=2 << 44, k_scale_dev=3 << 44, v_scale_dev=4 << 44)
    for prefix_len in (0, 5):
        prefix = _cache(n_heads=65535, head_dim=4, max_pos=5, sequences=1) if prefix_len else None
        args = B.make_attn8_args(P, P, P, P, P, P, P, _cache(n_heads=65535, head_dim=4, max_pos=1, sequences=1024, **far), 65535, prefix, prefix_len)
        assert _st(B.bl_attn8_decode, args) == B.BL_ERR_SHAPE
    assert _st(B.bl_attn8_prefill, P, P, P, P, P, P, _cache(n_heads=65535, head_dim=4, max_pos=65535), 65535, 0, 0, 65535) == B.BL_ERR_SHAPE


def _program(tmp_path, name, text):
    src = tmp_path / (name + ".cpp")
    src.write_text(text)
    exe = str(tmp_path / name)
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_2410_16144_amd", "csrc"), str(src), "-o", exe])
    return subprocess.run([exe]).returncode


def test_plan_covers_every_row_and_fits_its_merge(tmp_path):
    """For shapes over the whole range: at most 64 workgroups share a row's walk, every row is in a block, no workgroup is without positions
    of the longest walk, and a launch has more workgroups than it aims at only where its parts cannot be larger."""
    assert _program(tmp_path, "plan", """
        #include <initializer_list>
        #include "bl_attn8_plan.hpp"
        int main() {
            const int lens[] = {0, 1, 64, 127, 128, 129, 256, 257, 1000, 8001, 65536, 100003, 4194240};
            for (int heads : {1, 2, 7, 8, 32, 40, 64, 300})
                for (int group : {1, 2, 4, 5, 8, 16, 21, 64})
                    for (int tokens : {1, 2, 3, 8, 37, 64, 1024})
                        for (int shared : lens)
                            for (int own : lens) {
                                if (!shared && !own) continue;
                                const bl::Attn8Plan p = bl::attn8_plan(heads, group, tokens, shared, own, 16 * (1 + (heads + shared + own) % 16));
                                const int64_t rows = (int64_t)tokens * group;
                                if (p.block != 4 && p.block != 8 && p.block != 16) return 1;
                                if (p.tiles && (p.block != 4 || rows <= bl::kRows8Most || !shared)) return 10;
                                if ((shared > 0) != (p.shared_splits > 0) || (own > 0) != (p.own_splits > 0)) return 2;
                                if (p.shared_splits > 64 || p.own_splits > 64) return 3;
                                const int block = p.tiles ? p.tile_rows : p.block;
                                if (p.tile_rows > 32 && (!p.tiles || own || p.shared_splits != 1)) return 13;
                                if (shared && ((int64_t)p.shared_blocks * block < rows || (int64_t)(p.shared_blocks - 1) * block >= rows)) return 4;
                                if (own && p.own_blocks * p.block < group) return 5;
                                if (p.shared_splits > bl::sets_of(shared, p.shared_set) || p.own_splits > bl::sets_of(own, p.own_set)) return 6;
                                if (p.shared_set != (p.tiles ? (p.tile_rows == 128 ? 5 : p.tile_rows == 64 ? 6 : 7) : p.own_set) || p.own_set != (p.waves == 8 ? 9 : p.waves == 4 ? 8 : 7)) return 7;
                                if (p.waves != 8 && p.waves != (p.block == 4 && (!p.tiles || p.apart) ? 2 : 4)) return 12;
                                if ((p.tiles && !p.apart && p.waves != 4) || (p.apart && !p.tiles)) return 15;
                                const int64_t turns = p.folded ? (p.shared_blocks + 1) / 2 : p.shared_blocks;
                                if (p.shared_wgs % 8 || p.shared_units % 8 || p.shared_wgs < heads * p.shared_splits * turns || p.shared_wgs % (p.shared_units ? p.shared_units : 1)) return 8;
                                if (p.strips > 1 && (!p.tiles || own)) return 20;
                                if (p.strips != 1 && p.strips != 2 && p.strips != 4 && p.strips != 8) return 17;
                                if (shared && p.shared_wgs >= heads * p.shared_splits * turns + 8 * turns && p.strips == 1) return 18;
                                if (p.strips > 1 && p.shared_wgs >= heads * p.shared_splits * (turns + p.strips)) return 19;
                                if (p.folded && (!p.tiles || own || p.shared_splits != 1 || heads * turns * 4 < bl::kAttn8Waves)) return 16;
                                if (p.own_wgs != (int64_t)heads * tokens * p.own_blocks * p.own_splits) return 9;
                                const int64_t a = (int64_t)heads * p.shared_splits * p.shared_blocks * (p.tiles ? 4 : p.waves), b = p.own_wgs * p.waves;
                                const bool least = p.own_splits == 1 && a <= bl::kAttn8SharedWaves;   // the shared walk's share beside many own ones
                                if (!p.apart && a + b > bl::kAttn8Waves && (p.shared_splits > 1 || p.own_splits > 1) && !least) return 11;
                                if (p.apart && ((a > bl::kAttn8Waves && p.shared_splits > 1) || (b > bl::kAttn8Waves && p.own_splits > 1))) return 14;
                            }
            return 0;
        }""") == 0


def test_division_by_known_numbers(tmp_path):
    """Every quotient of numbers up to 2^31 - 1 near the multiples of a divisor, for divisors over the whole range."""
    assert _program(tmp_path, "divide", """
        #include "bl_attn8_plan.hpp"
        int main() {
            for (int64_t d = 1; d < (1ll << 31); d += d < 3000 ? 1 : d / 7 + 1) {
                const bl::Divider by = bl::divider((int)d);
                const int64_t most = ((1ll << 31) - 1) / d;
                for (int64_t q = 0; q <= most; q += 1 + q / 3 + (q > most / 2 ? most / 40 : 0))
                    for (int64_t n = q * d - 2; n <= q * d + 2; ++n)
                        if (n >= 0 && n < (1ll << 31) && bl::divided((int)n, by) != n / d) return 1;
                for (int64_t n = (1ll << 31) - 1; n > (1ll << 31) - 60; --n)
                    if (bl::divided((int)n, by) != n / d) return 2;
            }
            return 0;
        }""") == 0
