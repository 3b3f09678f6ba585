"""Append with rotation on host-only caches: the bookkeeping of pe_append_kv_batch, and what is refused before any state
changes; differential attention and rotation need a device."""
import ctypes
import random

import pytest

import paper_2609_04875_gb300 as pe
from paper_2609_04875_gb300 import binding


def pair(bits):
    return [pe.PagedKVCache(2, 2, 64, 16, 40, 6, 20, host_only=True, kv_bits=bits) for _ in range(2)]


def books(c, seqs):
    return c.free_list(), c.page_refs(), [(c.seq_info(s), c.page_table(s)) for s in seqs]


@pytest.mark.parametrize("bits", [16, 8])
def test_the_books_are_those_of_append(bits):
    rng = random.Random(bits)
    rope = pe.Rope([1.0, 0.1])
    for _ in range(20):
        a, b = pair(bits)
        seqs = [a.seq_create() for _ in range(3)]
        assert seqs == [b.seq_create() for _ in range(3)]
        for _ in range(12):
            if rng.random() < 0.2 and len(seqs) < 6:
                s = rng.choice(seqs)
                seqs.append(a.seq_fork(s))
                assert b.seq_fork(s) == seqs[-1]
            elif rng.random() < 0.3:
                s = rng.choice(seqs)
                tau = rng.randint(1, a.seq_info(s)[0] + 1)
                assert a.crop(s, tau) == b.crop(s, tau)
            else:
                some = rng.sample(seqs, rng.randint(1, len(seqs)))
                cu = [0]
                for _ in some:
                    cu.append(cu[-1] + rng.randint(0, 40))
                fails = []
                for call in (lambda: a.append_kv_batch(some, None, None, cu),
                             lambda: b.append_kv_rope_batch(some, None, None, cu, rope)):
                    try:
                        call()
                        fails.append(None)
                    except pe.PEError as e:
                        fails.append(e.kind)
                assert fails[0] == fails[1]
            assert books(a, seqs) == books(b, seqs)


def raw(cache, seq, rope, n=4, positions=None, Q=None, Q_out=None, heads=2):
    cu = binding.i32_array([0, n])
    return binding.lib().pe_append_kv_rope_batch(cache.handle, 1, binding.i32_array([seq]), None, None, cu, rope, positions, Q,
                                                 Q_out, heads, None)


def test_refusals_leave_the_books():
    cache = pair(16)[0]
    s = cache.seq_create()
    before = books(cache, [s])
    ok = pe.Rope([1.0])
    for rope in (None, pe.Rope([])._ref, pe.Rope([0.5] * 33)._ref, pe.Rope([float("inf")])._ref, pe.Rope([1.0], axis=[8])._ref,
                 pe.Rope([1.0], axis=[-1])._ref, pe.Rope([1.0], scale=float("nan"))._ref):
        assert raw(cache, s, rope) == -1
        assert books(cache, [s]) == before
    assert raw(cache, s, ok._ref, positions=2) == -1          # misaligned
    assert raw(cache, 3, ok._ref) == -1
    assert raw(cache, s, ok._ref, n=1000) == -2
    assert books(cache, [s]) == before
    null = binding._Rope(1, 0, 1, 1.0, None, None)
    assert raw(cache, s, ctypes.byref(null)) == -1
    assert raw(cache, s, ok._ref) == 0 and cache.seq_info(s) == (4, 4)


def test_device_calls_on_a_host_only_cache():
    cache = pair(16)[0]
    s = cache.seq_create()
    cache.append_kv(s, n_tokens=4)
    lib, one, cu = binding.lib(), binding.i32_array([s]), binding.i32_array([0, 2])
    rope = pe.Rope([1.0])
    assert lib.pe_rotate_batch(cache.handle, 1, one, 16, cu, 16, 1, 2, rope._ref, None, None) == -5
    assert lib.pe_rotate_batch(cache.handle, 1, one, 16, cu, 16, 1, 0, rope._ref, None, None) == -1
    assert lib.pe_rotate_batch(cache.handle, 1, one, 16, cu, 16, -1, 2, rope._ref, None, None) == -1
    assert lib.pe_rotate_batch(cache.handle, 1, one, 16, binding.i32_array([0, 5]), 16, 1, 2, rope._ref, None, None) == -2
    assert lib.pe_rotate_batch(cache.handle, 1, one, 16, binding.i32_array([0, 0]), 16, 1, 2, rope._ref, None, None) == 0
    assert lib.pe_rotate_batch(cache.handle, 1, None, 16, cu, 16, 1, 2, rope._ref, None, None) == -1
    assert lib.pe_rotate_batch(None, 1, one, 16, cu, 16, 1, 2, rope._ref, None, None) == -1
    assert lib.pe_diff_attn_batch(cache.handle, 1, one, 0, 16, cu, 32, 4, 0.1, 64, None, 1e-5, None) == -5
    assert lib.pe_diff_attn_batch(None, 1, one, 0, 16, cu, 32, 4, 0.1, 64, None, 1e-5, None) == -1
    assert "host-only" in lib.pe_last_error().decode() or "null" in lib.pe_last_error().decode()
    with pytest.raises(TypeError):
        cache.append_kv_rope_batch([s], None, None, [0, 1], 3)
    with pytest.raises(ValueError):
        pe.Rope([1.0, 2.0], axis=[0])
