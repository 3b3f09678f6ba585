"""What rotated appends leave in an 8-bit cache at the tokens' own positions, over several launches and in forks; frequencies of
either sign and of more than a radian; outputs side by side with their inputs."""
import pytest
import torch

import rope_diff_model as model
from test_gpu_rope import CASES, cu_of, filled, freqs, gen, position_table, randn

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")


def own_positions(kept, counts, axes=1):
    return torch.tensor([[a + j for a, n in zip(kept, counts) for j in range(n)]] * axes, device="cuda", dtype=torch.int32)


def check_pages(cache, seq, before, K, err, V, kept, ps):
    """Sequence `seq`, which held `before` (K, V of `kept` tokens) and got K (fp64, off by err at most) and V: pages before the
    partly filled one as they were, each value of the others rounded once to its page's codes (launches are cut between pages)."""
    now = cache.read_kv(seq)
    for name, held, new, e in (("K", 0, K, err), ("V", 1, V.double(), torch.zeros_like(V).double())):
        x = torch.cat([before[held].double(), new], dim=1)
        e = torch.cat([torch.zeros_like(before[held]).double(), e], dim=1)
        got, first = now[held].double(), kept // ps * ps
        assert got.shape == x.shape and torch.equal(got[:, :first], x[:, :first])
        pad = -(x.shape[1] - first) % ps
        page, g8, e = [torch.nn.functional.pad(t[:, first:], (0, 0, 0, 0, 0, pad)).unflatten(1, (-1, ps)) for t in (x, got, e)]
        scale = model.page_scale(page.abs().amax(dim=(2, 4), keepdim=True))
        step = torch.maximum(model.E8 * page.abs(), scale * 2.0 ** -10)
        excess = ((g8 - page).abs() - step * (1 + 1e-6) - 2 * e).max().item()
        assert excess <= 0, (name, seq, excess)


@pytest.mark.parametrize("d,ps,hkv,hq,L,counts,kept,pairs,inter,axis", CASES)
def test_8_bit_append_at_the_tokens_own_positions(d, ps, hkv, hq, L, counts, kept, pairs, inter, axis):
    g = gen(5 * d + ps + hq)
    cache, seqs, _, _ = filled(L, hkv, d, ps, kept, counts, bits=8, g=g)
    N, cu = sum(counts), cu_of(counts)
    K, V, Q = randn(g, L, N, hkv, d) * 3, randn(g, L, N, hkv, d), randn(g, L, N, hq, d)
    before = [cache.read_kv(s) for s in seqs]
    rope = pe.Rope(freqs(pairs), axis=axis, interleaved=inter, scale=0.75)
    out = cache.append_kv_rope_batch(seqs, K, V, cu, rope, Q=Q)
    pos = own_positions(kept, counts, rope.n_axes)
    model.check_rotated(out, *model.rotated(Q, pos, freqs(pairs), axis, inter, 0.75))
    want, err = model.rotated(K, pos, freqs(pairs), axis, inter, 0.75)
    for i, s in enumerate(seqs):
        check_pages(cache, s, before[i], want[:, cu[i]:cu[i + 1]], err[:, cu[i]:cu[i + 1]], V[:, cu[i]:cu[i + 1]], kept[i], ps)


@pytest.mark.parametrize("given", [False, True])
def test_8_bit_append_of_several_launches(given):
    g = gen(21)
    kept, counts = [3 + i % 5 for i in range(70)], [9 + i % 30 for i in range(70)]
    counts[5] = 26000  # more pages than one launch carries
    cache, seqs, _, _ = filled(2, 2, 64, 8, kept, counts, bits=8, g=g)
    N, cu = sum(counts), cu_of(counts)
    K, V = randn(g, 2, N, 2, 64), randn(g, 2, N, 2, 64)
    before = [cache.read_kv(s) for s in seqs]
    pos = position_table(1, N, g, far=False) if given else None
    launches = cache.kernel_launches()
    cache.append_kv_rope_batch(seqs, K, V, cu, pe.Rope(freqs(32)), positions=pos)
    assert cache.kernel_launches() - launches > 1
    want, err = model.rotated(K, pos if given else own_positions(kept, counts), freqs(32))
    for i, s in enumerate(seqs):
        check_pages(cache, s, before[i], want[:, cu[i]:cu[i + 1]], err[:, cu[i]:cu[i + 1]], V[:, cu[i]:cu[i + 1]], kept[i], 8)


def test_8_bit_append_after_a_fork():
    g = gen(22)
    cache, (s,), _, _ = filled(2, 2, 64, 16, [21], [64], bits=8, g=g, slack=16)
    f = cache.seq_fork(s)
    before = [t.clone() for t in cache.read_kv(s)]
    for seq in (f, s):
        K, V = randn(g, 2, 7, 2, 64) * 2, randn(g, 2, 7, 2, 64)
        cache.append_kv_rope(seq, K, V, pe.Rope(freqs(32)))
        want, err = model.rotated(K, own_positions([21], [7]), freqs(32))
        check_pages(cache, seq, before, want, err, V, 21, 16)


@pytest.mark.parametrize("bits", [16, 8])
def test_frequencies_of_either_sign_and_of_more_than_a_radian(bits):
    """Also whole turns and more; positions of either sign, as far as the model's products in 64 bits are exact enough."""
    g = gen(23)
    f = [-0.37, 3.0, -3.0, 6.5, -100.25, 0.0, -1e-4, 1e-9, 12345.678, 0.5, -0.5, 2.0, -2.0, 1.0, -1.0, 7.0]
    cache, (s,), _, _ = filled(1, 2, 64, 16, [5], [80], bits=bits, g=g)
    K, V, Q = randn(g, 1, 64, 2, 64), randn(g, 1, 64, 2, 64), randn(g, 1, 64, 4, 64)
    pos = torch.randint(-1000, 1000, (1, 64), generator=g, device="cuda", dtype=torch.int32)
    before = cache.read_kv(s)
    for inter in (False, True):
        rope = pe.Rope(f, interleaved=inter)
        model.check_rotated(cache.rotate_batch([s], Q, [0, 64], rope, positions=pos), *model.rotated(Q, pos, f, interleaved=inter))
    rq = cache.append_kv_rope(s, K, V, pe.Rope(f), Q=Q, positions=pos)
    model.check_rotated(rq, *model.rotated(Q, pos, f))
    want, err = model.rotated(K, pos, f)
    if bits == 8:
        check_pages(cache, s, before, want, err, V, 5, 16)
    else:
        model.check_rotated(cache.read_kv(s)[0][:, 5:], want, err)


def test_outputs_side_by_side_with_their_inputs():
    g = gen(24)
    cache, (s,), _, _ = filled(1, 2, 64, 16, [5], [40], g=g)
    rope = pe.Rope(freqs(32))
    both = randn(g, 2, 4, 2, 64)
    K = randn(g, 1, 4, 2, 64)
    Q = both[:1].clone()
    out = cache.append_kv_rope(s, K, K.clone(), rope, Q=both[:1], Q_out=both[1:])
    assert out.data_ptr() == both[1:].data_ptr() and torch.equal(both[:1], Q)
    model.check_rotated(out, *model.rotated(Q, own_positions([5], [4]), freqs(32)))
    x = cache.rotate(s, both[:1], rope, out=both[1:])
    assert torch.equal(x, out) and torch.equal(both[:1], Q)
