"""Rotation on the way into the cache and alone, against 64 bits."""
import pytest
import torch

import rope_diff_model as model

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda").to(torch.bfloat16)


def freqs(n, base=10000.0):
    return [base ** (-i / n) for i in range(n)]


def cu_of(counts):
    cu = [0]
    for n in counts:
        cu.append(cu[-1] + n)
    return cu


def filled(L, hkv, d, ps, kept, extra, bits=16, g=None, slack=4, **kw):
    """A cache whose sequences hold `kept` tokens, with room for `extra` more each."""
    per = max(-(-(a + b) // ps) for a, b in zip(kept, extra)) + 1
    cache = pe.PagedKVCache(L, hkv, d, ps, sum(-(-(a + b) // ps) for a, b in zip(kept, extra)) + slack, len(kept) + 2, per,
                            kv_bits=bits, **kw)
    seqs = [cache.seq_create() for _ in kept]
    N = sum(kept)
    K, V = randn(g, L, N, hkv, d), randn(g, L, N, hkv, d)
    cache.append_kv_batch(seqs, K, V, cu_of(kept))
    return cache, seqs, K, V


# d, ps, hkv, hq, L, counts appended, kept before, pairs, interleaved, axes
CASES = [
    (64, 16, 8, 8, 1, [1], [640], 32, False, None),
    (128, 16, 8, 32, 2, [1, 1, 1], [0, 15, 16], 64, False, None),
    (128, 8, 2, 4, 1, [7, 0, 33, 1], [5, 3, 0, 8], 64, True, None),
    (64, 128, 4, 8, 3, [129, 250], [1, 127], 8, False, [0] * 3 + [1] * 2 + [2] * 3),
    (64, 32, 3, 5, 2, [40, 9], [31, 70], 5, False, None),
    (128, 64, 1, 1, 1, [65, 2, 3], [63, 1, 64], 1, True, None),
    (128, 32, 2, 6, 2, [31, 100], [0, 33], 16, True, [i % 3 for i in range(16)]),
    (128, 16, 4, 8, 1, [300, 17], [2, 9], 24, False, [0] * 10 + [1] * 14),
    (64, 16, 2, 2, 1, [20], [3], 31, True, None),
    (64, 16, 5, 7, 2, [3] * 20, [i for i in range(20)], 16, False, None),
    (128, 128, 8, 8, 1, [400], [100], 64, False, None),
    (64, 8, 1, 3, 1, [1030], [2], 32, False, None),
]


def position_table(axes, N, g, far=True):
    hi = 2 ** 31 - 1 if far else 5000
    return torch.randint(-hi, hi, (axes, N), generator=g, device="cuda", dtype=torch.int32)


@pytest.mark.parametrize("given", [False, True])
@pytest.mark.parametrize("d,ps,hkv,hq,L,counts,kept,pairs,inter,axis", CASES)
def test_append_rotates_k_and_q_and_copies_v(d, ps, hkv, hq, L, counts, kept, pairs, inter, axis, given):
    g = gen(d + ps + hq)
    cache, seqs, K0, V0 = filled(L, hkv, d, ps, kept, counts, g=g)
    N, cu = sum(counts), cu_of(counts)
    K, V, Q = randn(g, L, N, hkv, d), randn(g, L, N, hkv, d), randn(g, L, N, hq, d)
    rope = pe.Rope(freqs(pairs), axis=axis, interleaved=inter, scale=1.25)
    axes = rope.n_axes
    pos = torch.tensor([[a + j for a, n in zip(kept, counts) for j in range(n)]] * axes, device="cuda", dtype=torch.int32)
    if given:
        pos = position_table(axes, N, g, far=False)
    before = Q.clone()
    out = cache.append_kv_rope_batch(seqs, K, V, cu, rope, Q=Q, positions=pos if given else None)
    assert [cache.seq_info(s)[0] for s in seqs] == [a + n for a, n in zip(kept, counts)]
    assert torch.equal(Q, before)
    model.check_rotated(out, *model.rotated(Q, pos, freqs(pairs), axis, inter, 1.25))
    want, err = model.rotated(K, pos, freqs(pairs), axis, inter, 1.25)
    cu0 = cu_of(kept)
    for i, s in enumerate(seqs):
        k, v = cache.read_kv(s)
        assert torch.equal(k[:, :kept[i]], K0[:, cu0[i]:cu0[i + 1]]) and torch.equal(v[:, :kept[i]], V0[:, cu0[i]:cu0[i + 1]])
        assert torch.equal(v[:, kept[i]:], V[:, cu[i]:cu[i + 1]])
        model.check_rotated(k[:, kept[i]:], want[:, cu[i]:cu[i + 1]], err[:, cu[i]:cu[i + 1]])
        assert torch.equal(k[:, kept[i]:, :, 2 * pairs:], K[:, cu[i]:cu[i + 1], :, 2 * pairs:])
        assert cache.device_page_table(s, len(cache.page_table(s))) == cache.page_table(s)
    # the queries' rotation alone gives the same bits; in place too
    again = cache.rotate_batch(seqs, Q, cu, rope, positions=pos if given else None)
    assert torch.equal(again, out)
    assert cache.rotate_batch(seqs, Q, cu, rope, positions=pos if given else None, out=Q) is Q
    assert torch.equal(Q, out)


@pytest.mark.parametrize("d,ps,hkv,hq,L,counts,kept,pairs,inter,axis", CASES)
def test_append_to_an_8_bit_cache_rounds_the_rotated_value_once(d, ps, hkv, hq, L, counts, kept, pairs, inter, axis):
    g = gen(3 * d + ps + hq)
    cache, seqs, _, _ = filled(L, hkv, d, ps, kept, counts, bits=8, g=g)
    N, cu = sum(counts), cu_of(counts)
    K, V, Q = randn(g, L, N, hkv, d) * 3, randn(g, L, N, hkv, d), randn(g, L, N, hq, d)
    before = [cache.read_kv(s) for s in seqs]
    rope = pe.Rope(freqs(pairs), axis=axis, interleaved=inter)
    pos = position_table(rope.n_axes, N, g, far=False)
    out = cache.append_kv_rope_batch(seqs, K, V, cu, rope, Q=Q, positions=pos)
    model.check_rotated(out, *model.rotated(Q, pos, freqs(pairs), axis, inter))
    want, err = model.rotated(K, pos, freqs(pairs), axis, inter)
    for i, s in enumerate(seqs):
        for name, held, new, e in (("K", 0, want[:, cu[i]:cu[i + 1]], err[:, cu[i]:cu[i + 1]]),
                                   ("V", 1, V[:, cu[i]:cu[i + 1]].double(), torch.zeros(1, device="cuda"))):
            x = torch.cat([before[i][held].double(), new], dim=1)
            e = torch.cat([torch.zeros_like(before[i][held]).double(), e.expand_as(new)], dim=1)
            got = cache.read_kv(s)[held].double()
            first = kept[i] // ps * ps
            assert torch.equal(got[:, :first], x[:, :first])
            for p0 in range(first, x.shape[1], ps):
                page, g8, pe_ = x[:, p0:p0 + ps], got[:, p0:p0 + ps], e[:, p0:p0 + ps]
                scale = model.page_scale(page.abs().amax(dim=(1, 3), keepdim=True))
                step = torch.maximum(model.E8 * page.abs(), scale * 2.0 ** -10)
                excess = ((g8 - page).abs() - step * (1 + 1e-6) - 2 * pe_).max().item()
                assert excess <= 0, (name, i, p0, excess)


def test_far_positions_keep_their_angles():
    """Angles of 2^31 positions times a radian."""
    g = gen(5)
    cache, seqs, _, _ = filled(1, 1, 128, 16, [4], [0], g=g)
    X = randn(g, 64, 3, 128)
    pos = position_table(1, 64, g)
    f = [1.0 / 4 ** i for i in range(13)] + [-0.37, 3.0]
    # in integers: a frequency that is a whole number of 2^-24 turns is exact in both
    turns = [round(x * 2 ** 24) for x in (0.3, 0.001, 0.7, 1.5)]
    rope = pe.Rope([t / 2 ** 24 * 6.283185307179586 for t in turns])
    out = cache.rotate_batch(seqs, X, [0, 64], rope, positions=pos)
    phase = (pos[0].long()[:, None] * torch.tensor(turns, device="cuda")) % 2 ** 24
    one = torch.arange(64, device="cuda")[None]
    y, e = X.double().clone(), torch.zeros_like(X.double())
    angle = (phase.double() / 2 ** 24 * 6.283185307179586)[:, None]
    a, b = y[..., 0:4].clone(), y[..., 4:8].clone()
    y[..., 0:4], y[..., 4:8] = a * angle.cos() - b * angle.sin(), b * angle.cos() + a * angle.sin()
    # (2 pi t as a double is off by 2^-53 of it: times 2^31 positions, 2^-20 radians or so)
    e[..., :8] = (a.abs() + b.abs()).repeat(1, 1, 2) * (2.0 ** -20 + 2.0 ** -18)
    model.check_rotated(out, y, e)
    assert one.numel() == 64 and len(f) == 15


def test_infinities_stay_in_their_pairs():
    g = gen(6)
    cache, seqs, _, _ = filled(1, 2, 64, 16, [3], [40], g=g)
    K, V, Q = randn(g, 1, 20, 2, 64), randn(g, 1, 20, 2, 64), randn(g, 1, 20, 4, 64)
    clean = cache.seq_fork(seqs[0])
    rope = pe.Rope(freqs(8))
    q0 = cache.append_kv_rope(clean, K, V, rope, Q=Q)
    k0, v0 = cache.read_kv(clean)
    K[0, 4, 1, 2], K[0, 5, 0, 60], Q[0, 7, 3, 9], V[0, 9, 0, 0] = float("inf"), float("nan"), float("-inf"), float("inf")
    q1 = cache.append_kv_rope(seqs[0], K, V, rope, Q=Q)
    k1, v1 = cache.read_kv(seqs[0])
    same = torch.ones_like(k0, dtype=torch.bool)
    same[0, 3 + 4, 1, 2] = same[0, 3 + 4, 1, 10] = same[0, 3 + 5, 0, 60] = False
    assert torch.equal(k1[same], k0[same]) and not torch.isfinite(k1[~same]).any()
    same = torch.ones_like(q0, dtype=torch.bool)
    same[0, 7, 3, 1] = same[0, 7, 3, 9] = False
    assert torch.equal(q1[same], q0[same]) and not torch.isfinite(q1[~same]).any()
    same = torch.ones_like(v0, dtype=torch.bool)
    same[0, 3 + 9, 0, 0] = False
    assert torch.equal(v1[same], v0[same]) and v1[0, 12, 0, 0] == float("inf")


def test_an_8_bit_cache_holds_such_tokens_as_nan():
    g = gen(7)
    cache, seqs, _, _ = filled(1, 2, 64, 16, [3], [40], bits=8, g=g)
    K, V = randn(g, 1, 20, 2, 64), randn(g, 1, 20, 2, 64)
    K[0, 4, 1, 2], V[0, 9, 0, 0] = float("inf"), float("nan")
    cache.append_kv_rope(seqs[0], K, V, pe.Rope(freqs(8)))
    k, v = cache.read_kv(seqs[0])
    bad = torch.zeros((23, 2), dtype=torch.bool, device="cuda")
    bad[7, 1] = bad[12, 0] = True
    assert torch.isnan(k[0][bad]).all() and torch.isnan(v[0][bad]).all()
    assert torch.isfinite(k[0][~bad]).all() and torch.isfinite(v[0][~bad]).all()


@pytest.mark.parametrize("bits", [16, 8])
def test_many_sequences_and_pages_take_several_launches(bits):
    g = gen(8)
    kept, counts = [3 + i % 5 for i in range(70)], [9 + i % 30 for i in range(70)]
    counts[5] = 26000  # more pages than one launch carries
    cache, seqs, _, _ = filled(1, 1, 64, 8, kept, counts, bits=bits, g=g)
    N, cu = sum(counts), cu_of(counts)
    K, V, Q = randn(g, 1, N, 1, 64), randn(g, 1, N, 1, 64), randn(g, 1, N, 2, 64)
    twin = pe.PagedKVCache(1, 1, 64, 8, cache.num_pages, 72, cache.max_pages_per_seq, kv_bits=bits)
    rope = pe.Rope(freqs(32))
    before = cache.kernel_launches()
    out = cache.append_kv_rope_batch(seqs, K, V, cu, rope, Q=Q)
    assert cache.kernel_launches() - before > 1
    pos = torch.tensor([[a + j for a, n in zip(kept, counts) for j in range(n)]], device="cuda", dtype=torch.int32)
    model.check_rotated(out, *model.rotated(Q, pos, freqs(32)))
    assert torch.equal(cache.rotate_batch(seqs, Q, cu, rope), out)
    twin.close()
    want, err = model.rotated(K, pos, freqs(32))
    if bits == 16:
        for i, s in enumerate(seqs):
            k, v = cache.read_kv(s)
            assert torch.equal(v[:, kept[i]:], V[:, cu[i]:cu[i + 1]])
            model.check_rotated(k[:, kept[i]:], want[:, cu[i]:cu[i + 1]], err[:, cu[i]:cu[i + 1]])


@pytest.mark.parametrize("bits", [16, 8])
def test_append_after_a_fork_copies_the_shared_page(bits):
    g = gen(9)
    cache, (s,), K0, V0 = filled(2, 2, 64, 16, [21], [64], bits=bits, g=g, slack=16)
    f = cache.seq_fork(s)
    held = [t.clone() for t in cache.read_kv(s)]
    K, V = randn(g, 2, 7, 2, 64), randn(g, 2, 7, 2, 64)
    cache.append_kv_rope(f, K, V, pe.Rope(freqs(32)))
    now = cache.read_kv(s)
    assert torch.equal(now[0], held[0]) and torch.equal(now[1], held[1])
    assert cache.page_table(f)[0] == cache.page_table(s)[0] and cache.page_table(f)[1] != cache.page_table(s)[1]
    if bits == 16:
        assert torch.equal(cache.read_kv(f)[0][:, :21], K0)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_failed_append_leaves_the_cache(bits):
    g = gen(10)
    cache, seqs, _, _ = filled(1, 2, 64, 8, [11, 12], [26000, 5], bits=bits, g=g)
    N = 26005
    K, V, Q = randn(g, 1, N, 2, 64), randn(g, 1, N, 2, 64), randn(g, 1, N, 2, 64)
    held = [[t.clone() for t in cache.read_kv(s)] for s in seqs]
    state = (cache.free_list(), [cache.page_table(s) for s in seqs], [cache.seq_info(s) for s in seqs])
    for k in range(0, 2 + (bits == 8)):
        cache.set_option("fail_launch_after", k)
        with pytest.raises(pe.PEError, match="injected"):
            cache.append_kv_rope_batch(seqs, K, V, [0, 26000, N], pe.Rope(freqs(32)), Q=Q)
        cache.set_option("fail_launch_after", -1)
        assert state == (cache.free_list(), [cache.page_table(s) for s in seqs], [cache.seq_info(s) for s in seqs])
        for s, h in zip(seqs, held):
            now = cache.read_kv(s)
            assert torch.equal(now[0], h[0]) and torch.equal(now[1], h[1])
            assert cache.device_page_table(s, 2) == cache.page_table(s)


def test_offsets_past_32_bits():
    """A pool of more than 2^32 elements, its last pages first; a tensor of more than 2^32 elements."""
    free, _ = torch.cuda.mem_get_info()
    if free < 60 << 30:
        pytest.skip("needs 60 GB")
    g = gen(11)
    pages = (1 << 32) // (2 * 16 * 128) + 64
    cache = pe.PagedKVCache(1, 2, 128, 16, pages, 2, 8, init_free_order=list(range(pages))[::-1])
    s = cache.seq_create()
    K, V = randn(g, 1, 50, 2, 128), randn(g, 1, 50, 2, 128)
    rope = pe.Rope(freqs(64))
    cache.append_kv_rope(s, K, V, rope)
    pos = torch.arange(50, device="cuda", dtype=torch.int32)[None]
    k, v = cache.read_kv(s)
    model.check_rotated(k, *model.rotated(K, pos, freqs(64)))
    assert torch.equal(v, V) and max(cache.page_table(s)) == pages - 1
    n = 1 << 19
    X = torch.zeros((1, n + 8, 64, 128), dtype=torch.bfloat16, device="cuda")
    X[0, -8:] = randn(g, 8, 64, 128)
    pos = torch.arange(n + 8, device="cuda", dtype=torch.int32)
    cache.rotate_batch([s], X, [0, n + 8], rope, positions=pos, out=X)
    tail = torch.Generator("cuda").manual_seed(11)
    for shape in ((1, 50, 2, 128), (1, 50, 2, 128)):
        randn(tail, *shape)
    model.check_rotated(X[0, -8:], *model.rotated(randn(tail, 8, 64, 128), pos[None, -8:], freqs(64)))
    assert not X[0, :1000].any()


def test_other_streams_graphs_and_two_calls():
    g = gen(12)
    cache, (s,), _, _ = filled(2, 2, 128, 16, [100], [40], g=g)
    K, V, Q = randn(g, 2, 20, 2, 128), randn(g, 2, 20, 2, 128), randn(g, 2, 20, 4, 128)
    rope = pe.Rope(freqs(64))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    q = cache.append_kv_rope(s, K, V, rope, Q=Q, stream=side)
    q2 = cache.rotate(s, Q, rope, stream=side)
    side.synchronize()
    pos = torch.arange(100, 120, device="cuda", dtype=torch.int32)[None]
    model.check_rotated(q, *model.rotated(Q, pos, freqs(64)))
    assert torch.equal(q, q2)
    # captured: replayed on other contents
    out, X, at = torch.empty_like(Q), Q.clone(), pos.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.rotate_batch([s], X, [0, 20], rope, positions=at, out=out)
    X.copy_(Q.flip(0))
    at.add_(1000)
    graph.replay()
    torch.cuda.synchronize()
    model.check_rotated(out, *model.rotated(Q.flip(0), pos + 1000, freqs(64)))


def test_empty_calls():
    cache = pe.PagedKVCache(1, 2, 64, 16, 8, 2, 4)
    s = cache.seq_create()
    rope = pe.Rope(freqs(32))
    e = torch.empty((1, 0, 2, 64), dtype=torch.bfloat16, device="cuda")
    before = cache.kernel_launches()
    assert cache.append_kv_rope(s, e, e, rope, Q=e).shape == e.shape
    assert cache.rotate(s, e, rope).shape == e.shape
    assert cache.append_kv_rope_batch([], e, e, [0], rope) is None
    assert cache.kernel_launches() == before and cache.seq_info(s) == (0, 0)


def test_refusals():
    g = gen(13)
    cache, (s,), _, _ = filled(1, 2, 64, 16, [5], [40], g=g)
    K = randn(g, 1, 4, 2, 64)
    rope = pe.Rope(freqs(32))
    state = cache.seq_info(s), cache.free_list()
    pos = torch.zeros((1, 4), dtype=torch.int32, device="cuda")
    both = randn(g, 2, 4, 2, 64)
    bad = [
        (dict(rope=None), TypeError), (dict(rope=pe.Rope([])), pe.PEError), (dict(rope=pe.Rope(freqs(33))), pe.PEError),
        (dict(rope=pe.Rope([float("nan")])), pe.PEError), (dict(rope=pe.Rope([1.0], axis=[8])), pe.PEError),
        (dict(rope=pe.Rope([1.0, 1.0], axis=[-1, 0])), pe.PEError), (dict(rope=pe.Rope([1.0], scale=float("inf"))), pe.PEError),
        (dict(positions=pos.long()), TypeError), (dict(positions=pos.cpu()), TypeError), (dict(positions=pos[:, :3]), ValueError),
        (dict(positions=torch.zeros((4, 2), dtype=torch.int32, device="cuda").t()[:1]), ValueError),
        (dict(Q=K[:, :3]), ValueError), (dict(Q=K.float()), TypeError), (dict(Q=K[0]), ValueError),
        (dict(Q=K.clone(), Q_out=K), pe.PEError), (dict(Q=both[:1], Q_out=both.flatten()[512:512 + 512].view(1, 4, 2, 64)), None),
        (dict(Q=both[:1], Q_out=both.flatten()[8:8 + 512].view(1, 4, 2, 64)), pe.PEError),
        (dict(Q=both[:1], Q_out=both.flatten()[514:514 + 512 - 2][:0].view(0, 4, 2, 64)), ValueError),
        (dict(Q_out=K.clone()), ValueError),
    ]
    for kw, err in bad:
        if err is None:
            continue
        args = dict(rope=rope) | kw
        with pytest.raises(err):
            cache.append_kv_rope_batch([s], K, K.clone(), [0, 4], **args)
        assert (cache.seq_info(s), cache.free_list()) == state, kw
    with pytest.raises(pe.PEError):
        cache.rotate(s, randn(g, 6, 2, 64), rope)            # more rows than the sequence has
    with pytest.raises(pe.PEError):
        cache.rotate(99, K, rope)
    x = randn(g, 5, 2, 64)
    with pytest.raises(pe.PEError):
        cache.rotate(s, x[:4], rope, out=x[1:])              # overlaps, but is not X
    with pytest.raises(ValueError):
        cache.rotate(s, randn(g, 4, 2, 32), rope)
    with pytest.raises(ValueError):
        cache.rotate(s, x[:, :, ::2].repeat(1, 1, 2)[:, ::1].transpose(0, 1), rope)
    with pytest.raises(ValueError):
        pe.Rope([1.0, 2.0], axis=[0])


def test_refuses_outputs_over_positions():
    g = gen(14)
    cache, (s,), _, _ = filled(1, 2, 64, 16, [5], [40], g=g)
    rope = pe.Rope(freqs(32), axis=[0] * 16 + [1] * 16)
    K = randn(g, 1, 4, 2, 64)
    both = torch.zeros(512 + 16, dtype=torch.bfloat16, device="cuda")
    X, pos = both[:512].view(1, 4, 2, 64), both[512:].view(torch.int32).view(2, 4)
    inside = both[496:512].view(torch.int32).view(2, 4)   # the last 32 bytes of X
    state = cache.seq_info(s), cache.free_list()
    with pytest.raises(pe.PEError, match="positions"):
        cache.append_kv_rope(s, K, K.clone(), rope, Q=X, Q_out=X, positions=inside)
    with pytest.raises(pe.PEError, match="positions"):
        cache.rotate(s, X, rope, positions=inside, out=X)
    assert (cache.seq_info(s), cache.free_list()) == state
    cache.rotate(s, X, rope, positions=pos, out=X)         # side by side
    cache.append_kv_rope(s, K, K.clone(), rope, Q=X, Q_out=X, positions=pos)
    assert cache.seq_info(s)[0] == 9
