"""Differential attention: infinities and NaN in V in some of several successive tiles on the causal edge.  A tile's keys that
are not finite are marked while others may still be at the tile before or after, so every pattern of marked and unmarked tiles
has to leave the rows before a bad key as they are."""
import pytest
import torch

from test_gpu_diff import Setup
from test_gpu_rope import cu_of

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")

BAD = [float("nan"), float("inf"), float("-inf")]
RUNS = 12  # of each call: all of them the same


def spoil(s, bad):
    """V of `bad` keys (of every sequence) not finite, one column of one kv-head each; the cache written anew."""
    V, at = s.V.clone(), cu_of(s.lens)
    for i, t in enumerate(bad):
        for b, n in enumerate(s.lens):
            if t < n:
                V[0, at[b] + t, (i + b) % s.hkv, (7 * t + i) % s.d] = BAD[i % 3]
    s.cache.crop_batch(s.seqs, [1] * len(s.seqs))
    s.cache.append_kv_batch(s.seqs, s.K, V, at)
    return V


def seen_bad(s, V, counts, hq):
    """bool [rows][Hq / 2]: rows that see a key whose V, of either kv-head of the pair, is not finite."""
    at, group, out = cu_of(s.lens), hq // s.hkv, []
    for b, (t, n) in enumerate(zip(s.lens, counts)):
        odd = (~torch.isfinite(V[0, at[b]:at[b + 1]])).any(dim=2).view(t, s.hkv // 2, 2).any(dim=2)
        out.append((odd.cumsum(dim=0) > 0)[t - n:].repeat_interleave(group, dim=1))
    return torch.cat(out)


def check(s, counts, hq, bad):
    q, lam, gain = s.inputs(counts, hq)
    cu = cu_of(counts)
    for g in (gain, None):
        want = s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=g)
        s.check(want, s.seqs, q, cu, lam, g)
        V = spoil(s, bad)
        hit = seen_bad(s, V, counts, hq)
        for _ in range(RUNS):
            got = s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=g)
            assert torch.equal(got[~hit], want[~hit])
            assert not torch.isfinite(got[hit]).all(dim=1).any()
            assert s.cache.device_status() == 0
        spoil(s, [])


# 60 queries, a row each: two tiles of 64 keys (or one) are on the block's edge
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,bad", [(200, [195]), (200, [150]), (200, [150, 195]), (185, [133, 184]), (1500, [1499]), (4100, [4070, 4099])])
def test_few_rows(T, bad, d):
    check(Setup([T], 2, d, 16, seed=T + d), [60], 2, bad)


@pytest.mark.parametrize("T,n,hq", [(300, 60, 16), (2500, 33, 16), (300, 15, 64)])
def test_few_rows_of_many_units(T, n, hq):
    """Sequences of their own lengths, so that some have their bad key in the second tile of the edge and some in the first."""
    lens = [T - 7 * i for i in range(12)]
    check(Setup(lens, 16, 64, 16, seed=T + n), [n] * 12, hq, [T - 90, T - 40, T - 5])


# 65 to 128 rows: two blocks of 64, each with its own edge; one query's 128 heads in both
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,n,hq,bad", [(700, 128, 2, [650, 699]), (5000, 100, 2, [4990]), (2000, 32, 8, [1985]), (130, 65, 2, [64, 129]),
                                        (300, 1, 256, [299]), (200, 128, 2, [100])])
def test_two_blocks(T, n, hq, bad, d):
    check(Setup([T], 2, d, 16, seed=T + n + hq), [n], hq, bad)


# tiles of 128 keys: a block of 256 rows has two or three on the edge, a whole prompt all of them
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,n,bad", [(700, 300, [690]), (700, 300, [450, 690]), (700, 700, [5]), (700, 700, [140, 300, 520]), (700, 700, [260, 699]),
                                     (3000, 280, [2999]), (3000, 600, [2500, 2900])])
def test_many_rows(T, n, bad, d):
    check(Setup([T], 4, d, 32, seed=T + n + d), [n], 8, bad)


def test_many_rows_of_many_units():
    lens = [600 - 11 * i for i in range(9)]
    check(Setup(lens, 8, 64, 16, seed=77), lens, 8, [130, 390, 585])


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("T,n,hq", [(200, 60, 2), (130, 60, 2), (330, 16, 8), (700, 300, 8), (385, 385, 8), (129, 129, 2)])
def test_slots_past_the_end(T, n, hq, d):
    """What a crop left in the slots behind a sequence, in the last tile of the edge alone, reaches no row."""
    s = Setup([T], 2, d, 128, seed=T + n + d)
    q, lam, gain = s.inputs([n], hq)
    want = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    s.check(want, s.seqs, q, [0, n], lam, gain)
    extra = 128 - T % 128 if T % 128 else 0
    rest = torch.full((1, extra, 2, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    s.cache.append_kv(s.seqs[0], rest, rest)
    s.cache.crop(s.seqs[0], T + 1)
    for _ in range(RUNS):
        assert torch.equal(s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain), want)
        assert s.cache.device_status() == 0
