"""The 8-bit cache on the GPU against its definition in 64 bits (q8_model.py): what append, crop, fork and eviction
leave in the cache (bit for bit), attention over it, the keys' accumulated weights, and what is refused.

Attention's bound, element by element: against the values held, the kernels differ from the exact result by the output's
rounding to bf16 (2^-8 |o|), the softmax weights' rounding (to bf16 or finer: 2^-8 of each, so 2^-8 sum_j w_j |v_j|) and
the scores' error as below, times the same sum; a twentieth is added for the products of these.  Weights held in e4m3
parts have an absolute floor too: n keys each off by 2^-24 of the largest, times the largest |v|.  The weights are fp32
sums of terms 2^(x - lse): an error dx of a score (a dot product of d exact products, each addition within 2^-24 of
the sum of magnitudes) moves a term by a factor 2^dx, lse's own error no further, the exponential and logarithm add
2^-20, and each of the sum's additions 2^-24."""
import math

import numpy as np
import pytest
import torch

import q8_model
import synth
from gpu_common import requires_cuda

pytestmark = [pytest.mark.gpu, requires_cuda]


def to64(t):
    return t.double().cpu().numpy()


def score_error(K, Q, scale):
    """In log2 units, at most: a score's own error and that of the row's reference."""
    mag = scale * math.log2(math.e) * np.abs(Q).max(axis=(0, 1)) @ np.abs(np.nan_to_num(K)).max(axis=(0, 1))
    return 2 * (Q.shape[-1] + 8) * 2.0 ** -24 * mag


def assert_attention(out, m, Q, scale, layer=0, what=""):
    """out against the model's attention of sequence m's last rows Q (64 bits); returns the keys' weights."""
    ref, w, size = q8_model.attend(m.K[layer], m.V[layer], Q, scale)
    floor = len(m) * 2.0 ** -24 * np.abs(np.nan_to_num(m.V[layer])).max()
    got = to64(out)
    assert np.array_equal(np.isnan(got), np.isnan(ref)), f"{what}: NaN rows"
    bound = 1.05 * (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + score_error(m.K[layer], Q, scale)) * size + floor)
    over = np.nan_to_num(np.abs(got - ref) / bound)
    assert over.max() <= 1, f"{what}: error {over.max():.3g} times the bound"
    return w


def bf16(x):
    """numpy -> bf16 CUDA tensor and its exact values in 64 bits."""
    t = torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16)
    return t.cuda(), t.double().numpy()


class Both:
    """A library cache and the model, driven together."""

    def __init__(self, L=1, hkv=2, d=64, ps=16, pages=64, seqs=8, seed=1, bits=8, max_pages=None, workspace=0):
        import paper_2609_04875_gb300 as pe
        self.dims = (L, hkv, d, ps)
        self.bits = bits
        self.cache = pe.PagedKVCache(L, hkv, d, ps, pages, seqs, max_pages or pages,
                                     init_free_order=synth.page_permutation(seed, pages), kv_bits=bits, workspace_bytes=workspace)
        self.seqs = {}
        self.g = np.random.default_rng(seed)

    def draw(self, n, spread=1.0):
        L, hkv, d, _ = self.dims
        x = self.g.standard_normal((L, n, hkv, d)) * np.exp(spread * self.g.standard_normal((L, n, hkv, 1)))
        return x.astype(np.float32)

    def new(self):
        s = self.cache.seq_create()
        self.seqs[s] = q8_model.Seq(*self.dims, bits=self.bits)
        return s

    def append(self, seqs, counts, k=None, v=None, spread=1.0):
        cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
        k, k64 = bf16(self.draw(cu[-1], spread) if k is None else k)
        v, v64 = bf16(self.draw(cu[-1], spread) if v is None else v)
        self.cache.append_kv_batch(seqs, k, v, cu)
        for i, s in enumerate(seqs):
            self.seqs[s].append(k64[:, cu[i]: cu[i + 1]], v64[:, cu[i]: cu[i + 1]])

    def crop(self, s, tau):
        self.cache.crop(s, tau)
        self.seqs[s].crop(tau)

    def fork(self, s):
        f = self.cache.seq_fork(s)
        self.seqs[f] = self.seqs[s].fork()
        return f

    def check(self):
        L, hkv, d, ps = self.dims
        for s, m in self.seqs.items():
            assert self.cache.seq_info(s)[0] == len(m)
            if len(m) == 0:
                continue
            k, v = self.cache.read_kv(s)
            np.testing.assert_array_equal(to64(k), m.K)
            np.testing.assert_array_equal(to64(v), m.V)
            if self.bits == 8:
                exps = self.scales()[:, self.cache.page_table(s)]
                np.testing.assert_array_equal(exps, m.E)
            assert self.cache.device_page_table(s, len(self.cache.page_table(s))) == self.cache.page_table(s)
        assert self.cache.device_status() == 0

    def scales(self):
        import ctypes
        from paper_2609_04875_gb300 import binding
        L, hkv, d, ps = self.dims
        ptr = ctypes.c_void_p()
        assert binding.lib().pe_cache_scales(self.cache.handle, ctypes.byref(ptr)) == 0
        shape = (L, self.cache.num_pages, hkv, 2)

        class Arr:  # the device array, through torch's view of a foreign buffer
            __cuda_array_interface__ = {"shape": shape, "typestr": "|i1", "data": (ptr.value, False), "version": 3}
        return torch.as_tensor(Arr(), device="cuda").cpu().numpy().astype(np.int64)


# ---------------------------------------------------------------- what the cache holds
@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("L,hkv,d", [(1, 1, 64), (2, 3, 128)])
def test_appends_of_every_kind(ps, L, hkv, d):
    b = Both(L, hkv, d, ps, pages=60)
    a, c = b.new(), b.new()
    b.append([a, c], [1, 0])                       # a single token, and none
    b.append([c, a], [ps, ps - 1])                 # a full page; the rest of one
    b.check()
    b.append([a, c], [2 * ps + 3, 5], spread=4.0)  # pages whose tokens differ in size by 2^10 and more
    for n in (1, 1, 2):
        b.append([a], [n], spread=4.0)             # onto a partly filled page: its scale may grow
    b.check()
    b.append([c], [2], k=b.draw(2) * 0, v=b.draw(2) * 0)  # zeros
    f = b.fork(a)
    b.append([f], [3], spread=6.0)                 # copy-on-write, then quantised again: the base stays as it is
    b.append([a], [2], spread=6.0)
    b.check()
    b.crop(a, ps + 2)                              # a page kept in part, its scale from tokens now gone
    b.check()
    b.append([a], [1], spread=0.1)
    b.check()
    b.crop(f, 1)
    b.append([f], [7])
    b.check()


def test_zero_tiny_huge_and_nonfinite_values():
    b = Both(1, 2, 64, 16)
    s = b.new()
    k, v = b.draw(40), b.draw(40)
    k[0, 0:16] *= 2.0 ** -120                      # below what e >= -126 reaches in full
    v[0, 0:16] *= 0
    k[0, 16:32] *= 2.0 ** 100
    v[0, 17] = 2.0 ** 127 * 1.99                   # past 448 * 2^119: held as that
    k[0, 33, 1, 5] = np.inf                        # kv-head 1 of token 33 only
    v[0, 35, 0, 63] = np.nan
    v[0, 36, 1, 0] = -np.inf
    b.append([s], [40], k, v)
    got = to64(b.cache.read_kv(s)[0])
    assert np.isnan(got[0, 33, 1]).all() and np.isfinite(got[0, 33, 0]).all()
    assert np.isnan(got[0, 35, 0]).all() and np.isnan(got[0, 36, 1]).all()
    m = b.seqs[s]
    held = np.maximum(np.abs(m.K), 2.0 ** -126)    # (bf16 holds smaller values with fewer bits)
    np.testing.assert_allclose(got, m.K, atol=2.0 ** -133, rtol=0)
    np.testing.assert_array_equal(np.where(held > 2.0 ** -126, got, 0), np.where(held > 2.0 ** -126, m.K, 0))
    np.testing.assert_array_equal(to64(b.cache.read_kv(s)[1]), m.V)


def test_long_appends_cut_over_launches():
    """More new pages than one launch carries, and more sequences."""
    b = Both(1, 1, 64, 8, pages=3400, seqs=80, max_pages=3300)
    s = b.new()
    b.append([s], [8 * 3200 + 5])
    many = [b.new() for _ in range(70)]
    b.append(many, [(i * 7) % 5 for i in range(70)])
    b.check()


def test_read_ranges_and_bf16_caches():
    for bits in (8, 16):
        b = Both(2, 2, 128, 16, bits=bits)
        s, t = b.new(), b.new()
        b.append([s, t], [50, 33])
        k, v = b.cache.read_kv_batch([t, s, s], [0, 17, 50], [0, 33, 50, 50])
        np.testing.assert_array_equal(to64(k), np.concatenate([b.seqs[t].K, b.seqs[s].K[:, 17:34]], 1))
        np.testing.assert_array_equal(to64(v), np.concatenate([b.seqs[t].V, b.seqs[s].V[:, 17:34]], 1))


def test_crop_and_replay_equal_from_scratch():
    """Theorem 1 on an 8-bit cache: the kept prefix and the replayed suffix are held as a fresh session is."""
    b = Both(1, 2, 64, 16)
    s, fresh = b.new(), b.new()
    k, v = b.draw(100, 0.3), b.draw(100, 0.3)
    b.append([s], [90])
    b.crop(s, 1)
    b.append([s], [70], k[:, :70], v[:, :70])
    b.append([s], [20], spread=0.3)
    b.crop(s, 71)
    b.append([s], [30], k[:, 70:], v[:, 70:])
    b.append([fresh], [100], k, v)
    b.check()
    np.testing.assert_array_equal(b.seqs[s].K, b.seqs[fresh].K)
    q = bf16(np.random.default_rng(3).standard_normal((30, 4, 64)))[0]
    assert torch.equal(b.cache.replay_attn(s, 0, q), b.cache.replay_attn(fresh, 0, q))


# ---------------------------------------------------------------- attention and the keys' weights
def weights_bound(K, Q, scale, w):
    """Per key: the scores' error as a factor, the exponential's, the sum's."""
    return w * (math.log(2) * score_error(K, Q, scale) + 2.0 ** -20 + Q.shape[0] * Q.shape[1] * 2.0 ** -24) + 1e-30


def run_attention(b, seqs, counts, hq, layer=0, scale=None, weights=True, q_scale=1.0, stride=None, pieces=1):
    L, hkv, d, ps = b.dims
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    q, q64 = bf16(b.g.standard_normal((cu[-1], hq, d)).astype(np.float32) * q_scale)
    scale = 1.0 / math.sqrt(d) if scale is None else scale
    out = b.cache.replay_attn_batch(seqs, layer, q, cu, softmax_scale=scale)
    longest = max(len(b.seqs[s]) for s in seqs)
    acc0 = torch.rand((len(seqs), stride or longest), device="cuda")
    if weights:
        full = torch.full((len(seqs), (stride or longest) + 5), 7.0, device="cuda")  # rows with a gap between them
        acc = full[:, : stride or longest]
        acc.copy_(acc0)
        out2 = b.cache.replay_attn_weights_batch(seqs, layer, q, cu, acc, softmax_scale=scale)
        again = acc0.clone()
        b.cache.replay_attn_weights_batch(seqs, layer, q, cu, again, softmax_scale=scale)
        assert torch.equal(torch.nan_to_num(acc, 1e9), torch.nan_to_num(again, 1e9))  # the order of the sums is fixed
        assert bool((full[:, acc.shape[1]:] == 7.0).all())
    assert b.cache.device_status() == 0
    for i, s in enumerate(seqs):
        m, n = b.seqs[s], counts[i]
        if n == 0:
            if weights:
                assert torch.equal(acc[i], acc0[i])
            continue
        w = assert_attention(out[cu[i]: cu[i + 1]], m, q64[cu[i]: cu[i + 1]], scale, layer, f"sequence {i}")
        if weights:
            assert_attention(out2[cu[i]: cu[i + 1]], m, q64[cu[i]: cu[i + 1]], scale, layer, f"sequence {i}, with weights")
            add = to64(acc[i, : len(m)]) - to64(acc0[i, : len(m)])
            bound = weights_bound(m.K[layer], q64[cu[i]: cu[i + 1]], scale, w) + pieces * 2.0 ** -24 * (1 + w)  # added that many times
            ok = ~np.isnan(w)
            assert np.array_equal(np.isnan(add), ~ok)
            assert (np.abs(add - w)[ok] <= bound[ok]).all(), f"sequence {i}: weights off by {np.abs(add - w)[ok].max():.3g}"
            assert torch.equal(acc[i, len(m):], acc0[i, len(m):])


@pytest.mark.parametrize("ps", [8, 16, 32, 64, 128])
@pytest.mark.parametrize("hq,hkv,d", [(1, 1, 64), (8, 2, 64), (16, 1, 128), (8, 1, 128), (4, 2, 128), (32, 1, 64)])
def test_single_tokens(ps, hq, hkv, d):
    b = Both(1, hkv, d, ps, pages=1400 // ps + 20)
    lens = [1, 2, ps, ps + 1, 127, 128, 129, 700]
    seqs = [b.new() for _ in lens]
    b.append(seqs, lens)
    run_attention(b, seqs, [1] * len(seqs), hq)


@pytest.mark.parametrize("n", [2, 3, 5, 16, 17, 40, 130])
@pytest.mark.parametrize("hq,hkv,d,ps", [(4, 2, 64, 16), (8, 1, 128, 8), (2, 2, 128, 64)])
def test_several_tokens(n, hq, hkv, d, ps):
    b = Both(2, hkv, d, ps, pages=1200 // ps + 20)
    lens = [n, n + 1, 300, 257]
    seqs = [b.new() for _ in lens]
    b.append(seqs, lens)
    run_attention(b, seqs, [n, n, 0, min(n, 257)], hq, layer=1)


def test_long_sessions_and_many_sequences():
    b = Both(1, 2, 128, 16, pages=2600, seqs=80)
    long_ = b.new()
    b.append([long_], [20011], spread=0.5)
    run_attention(b, [long_], [1], 8)
    run_attention(b, [long_], [3], 16)
    run_attention(b, [long_], [8], 16)
    many = [b.new() for _ in range(70)]
    b.append(many, [1 + (i * 37) % 200 for i in range(70)])
    run_attention(b, many, [1] * 70, 4)


@pytest.mark.parametrize("workspace", [1 << 15, 1 << 17, 1 << 20])
def test_small_workspaces(workspace):
    """Partials, kept scores and row groups that do not fit: fewer sequences a launch, a sequence's queries in pieces,
    or the unpacked layer; always the same results."""
    b = Both(1, 2, 64, 16, pages=250, workspace=workspace)
    seqs = [b.new() for _ in range(3)]
    b.append(seqs, [1500, 700, 40])
    for counts in ([1, 1, 1], [5, 1, 2], [40, 3, 40], [150, 0, 1]):
        run_attention(b, seqs, counts, 4, pieces=max(counts))


def test_windows_with_masked_and_nan_keys():
    """Many rows with weights: groups of rows that end inside a group, keys seen by some of them, NaN keys."""
    b = Both(1, 2, 128, 16, pages=80)
    s, t = b.new(), b.new()
    k, v = b.draw(700, 0.5), b.draw(700, 0.5)
    v[0, 690, 1, 3] = np.inf
    k[0, 3, 0, 0] = np.nan
    b.append([s], [700], k, v)
    b.append([t], [129])
    run_attention(b, [s, t], [20, 129], 4)
    run_attention(b, [t, s], [33, 300], 8)


@pytest.mark.parametrize("q_scale", [0.0, 8.0, 60.0])
def test_flat_and_peaked_scores(q_scale):
    """All scores equal; a few keys take everything (weights far below 2^-24 of the largest elsewhere)."""
    b = Both(1, 1, 128, 16, pages=200)
    s = b.new()
    b.append([s], [1500], spread=0.2)
    run_attention(b, [s], [1], 4, q_scale=q_scale)
    run_attention(b, [s], [9], 2, q_scale=q_scale)


def test_scores_that_rise_along_the_keys():
    """The softmax's reference moves in every tile; the last keys take everything."""
    b = Both(1, 1, 64, 16, pages=80)
    s = b.new()
    n = 1100
    k, v = b.draw(n, 0.0), b.draw(n, 0.0)
    k[0, :, 0, 0] = np.linspace(0, 60, n)
    b.append([s], [n], k, v)
    q = torch.zeros((1, 4, 64), device="cuda", dtype=torch.bfloat16)
    q[0, :, 0] = torch.tensor([1.0, 4.0, -2.0, 30.0])
    out = b.cache.replay_attn(s, 0, q, softmax_scale=1.0)
    assert_attention(out, b.seqs[s], to64(q), 1.0)


def test_pages_whose_values_differ_in_size():
    """V scales a factor 2^30 apart between pages, in the order that hurts: the small ones carry the weight."""
    b = Both(1, 1, 64, 16, pages=80)
    s = b.new()
    n = 512
    k, v = b.draw(n, 0.0), b.draw(n, 0.0)
    v[0, 100:116] *= 2.0 ** 15
    v[0, 300:316] *= 2.0 ** -15
    v[0, 320:336] *= 0
    k[0, 100:116, 0, 0] = -40
    k[0, 300:316, 0, 0] = 4
    b.append([s], [n], k, v)
    q = torch.zeros((1, 2, 64), device="cuda", dtype=torch.bfloat16)
    q[0, :, 0] = torch.tensor([1.0, 0.5])
    out = b.cache.replay_attn(s, 0, q, softmax_scale=1.0)
    assert_attention(out, b.seqs[s], to64(q), 1.0)


def test_nan_tokens_reach_only_the_rows_that_see_them():
    b = Both(1, 2, 64, 16)
    s = b.new()
    k, v = b.draw(140), b.draw(140)
    v[0, 136, 1, 3] = np.inf        # seen by the last four queries only, kv-head 1
    b.append([s], [140], k, v)
    run_attention(b, [s], [8], 4)
    run_attention(b, [s], [30], 4)
    # cropped away, its slot is stale on a page in use: no row may see it
    b.crop(s, 137)
    run_attention(b, [s], [1], 4)
    run_attention(b, [s], [20], 4)
    f = b.fork(s)
    b.append([f], [1])
    run_attention(b, [f], [1], 8)


@pytest.mark.parametrize("hq,hkv,n,d,ps", [(4, 2, 9, 128, 16), (8, 2, 13, 64, 8), (32, 1, 1, 128, 64), (16, 1, 4, 64, 128), (1, 1, 50, 128, 8),
                                           (8, 1, 16, 128, 32), (2, 1, 64, 128, 128), (16, 2, 9, 128, 16)])
def test_blocks_of_many_rows(hq, hkv, n, d, ps):
    """Blocks of 32, 64 and 128 rows, whole and not, with tiles that only some rows see; one launch also of few rows."""
    b = Both(1, hkv, d, ps, pages=26000 // ps + 20)
    lens = [8192 + n // 2, 2049, 12000, 1793, 130]
    seqs = [b.new() for _ in lens]
    b.append(seqs, lens, spread=0.5)
    run_attention(b, seqs, [n, n, n, 1, n], hq)


@pytest.mark.parametrize("hq,hkv,n,d,lens", [(128, 1, 1, 128, [17000, 300, 5]), (128, 1, 3, 64, [2000, 700]), (64, 1, 2, 128, [9000, 9000]),
                                             (32, 8, 16, 128, [1500] * 12), (4, 2, 13, 128, [100 + 3 * i for i in range(70)])])
def test_wide_groups_and_many_sequences(hq, hkv, n, d, lens):
    """A query of one sequence fills a block, or several; more sequences than a launch carries."""
    b = Both(1, hkv, d, 16, pages=sum(x // 16 + 1 for x in lens) + 40, seqs=80)
    seqs = [b.new() for _ in lens]
    b.append(seqs, lens, spread=0.5)
    run_attention(b, seqs, [min(n, x) for x in lens], hq)


@pytest.mark.parametrize("rows", [32, 64, 128])
@pytest.mark.parametrize("d", [64, 128])
def test_references_that_move_row_by_row(rows, d):
    """Scores that rise for some rows and fall for others, in steps below and above the slack of a block's references; a
    few tokens that outweigh all others, in different tiles for different rows."""
    b = Both(1, 1, d, 16, pages=540)
    s = b.new()
    n, g = 8300, 16
    k, v = b.draw(n, 0.0) * 0.1, b.draw(n, 0.0)
    k[0, :, 0, 0] = np.linspace(-80, 80, n)
    k[0, ::37, 0, 1] = 40 * b.g.standard_normal(len(range(0, n, 37)))
    b.append([s], [n], k, v)
    q = b.g.standard_normal((rows // g, g, d)).astype(np.float32) * 0.1
    q[..., 0] = np.linspace(-1.5, 1.5, rows).reshape(rows // g, g)
    q[..., 1] = np.where(np.arange(rows).reshape(rows // g, g) % 3 == 0, 3.0, 0.0)
    q, q64 = bf16(q)
    out = b.cache.replay_attn(s, 0, q, softmax_scale=1.0)
    assert b.cache.device_status() == 0
    assert_attention(out, b.seqs[s], q64, 1.0)


def test_many_rows_with_nan_tokens_and_scales_apart():
    """NaN tokens reach the rows that see them; V scales 2^30 apart; a row of q that is infinite or NaN stays alone."""
    b = Both(1, 2, 128, 16, pages=540)
    s = b.new()
    n = 8300
    k, v = b.draw(n, 0.3), b.draw(n, 0.3)
    v[0, 4000:4016] *= 2.0 ** 30
    k[0, 4000:4016] *= -4.0
    k[0, n - 9, 0, 5] = np.nan
    v[0, n - 20, 1, 0] = np.inf
    b.append([s], [n], k, v)
    q, q64 = bf16(b.g.standard_normal((31, 4, 128)).astype(np.float32))
    q[3, 1, 7] = float("inf")
    q[4, 2, 0] = float("nan")
    q64[3, 1], q64[4, 2] = np.nan, np.nan
    out = b.cache.replay_attn(s, 0, q)
    assert b.cache.device_status() == 0
    ref, w, size = q8_model.attend(b.seqs[s].K[0], b.seqs[s].V[0], q64, 1 / math.sqrt(128))
    got = to64(out)
    assert np.array_equal(np.isnan(got), np.isnan(ref))
    bound = 1.05 * (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + score_error(np.nan_to_num(b.seqs[s].K[0]), np.nan_to_num(q64), 1 / math.sqrt(128))) * size
                    + n * 2.0 ** -24 * np.abs(np.nan_to_num(b.seqs[s].V[0])).max())
    assert (np.nan_to_num(np.abs(got - ref) / bound) <= 1).all()


def test_stale_and_freed_slots_are_never_seen():
    b = Both(1, 2, 64, 16)
    b.cache.set_option("debug_poison", 1)
    s, t = b.new(), b.new()
    b.append([s, t], [200, 100])
    b.crop(s, 131)
    run_attention(b, [s, t], [1, 20], 4)
    b.append([s], [5])
    run_attention(b, [s, t], [5, 1], 4)
    b.check()


def test_rounds_and_static_scratch():
    """pe_replay_rounds and the static-scratch call on an 8-bit cache."""
    b = Both(2, 2, 64, 16)
    s = b.new()
    b.append([s], [77])
    k, k64 = bf16(b.draw(6))
    v, v64 = bf16(b.draw(6))
    q, q64 = bf16(b.g.standard_normal((2, 6, 4, 64)).astype(np.float32))
    out = b.cache.replay_rounds([s], np.array([[3], [1], [2]], dtype=np.int32), [0, 6], k, v, q)
    done = 0
    for take in (3, 1, 2):
        b.seqs[s].append(k64[:, done: done + take], v64[:, done: done + take])
        for layer in range(2):
            assert_attention(out[layer, done: done + take], b.seqs[s], q64[layer, done: done + take], 0.125, layer)
        done += take
    got = b.cache.replay_attn_static_scratch(s, 1, q[1])
    assert_attention(got, b.seqs[s], q64[1], 0.125, 1)


def test_another_stream():
    b = Both(1, 2, 64, 16)
    s = b.new()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.append([s], [333])
        run_attention(b, [s], [1], 8)
        w = torch.rand((1, 333), device="cuda")
        kept = b.cache.evict_batch([s], [100], w, sinks=2, recent=9)
    side.synchronize()
    assert int(kept[0, 0]) == 0 and kept.shape == (1, 100)


def test_weights_on_a_bf16_cache():
    b = Both(2, 2, 128, 16, bits=16)
    s, t = b.new(), b.new()
    b.append([s, t], [260, 40], spread=0.3)
    run_attention(b, [s, t], [1, 1], 8, layer=1)
    run_attention(b, [s, t], [33, 40], 4, layer=1)


# ---------------------------------------------------------------- eviction
def evict(b, seqs, keep, weights, sinks=0, recent=0):
    w = torch.from_numpy(weights).cuda()
    kept = b.cache.evict_batch(seqs, keep, w, sinks=sinks, recent=recent)
    got = kept.cpu().numpy()
    for i, s in enumerate(seqs):
        want, left = b.seqs[s].evict(keep[i], weights[i], sinks, recent)
        np.testing.assert_array_equal(got[i, : len(want)], want)
        assert (got[i, len(want):] == -1).all()
        np.testing.assert_array_equal(w[i].cpu().numpy(), left)
    b.check()


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("L,hkv,d,ps", [(1, 2, 64, 8), (2, 1, 128, 16), (1, 3, 64, 32), (2, 2, 128, 128)])
def test_eviction(bits, L, hkv, d, ps):
    b = Both(L, hkv, d, ps, pages=2200 // ps + 40, bits=bits)
    lens = [300, 1, 77, 600]
    seqs = [b.new() for _ in lens]
    b.append(seqs, lens, spread=2.0)
    w = b.g.exponential(size=(4, 640)).astype(np.float32)
    evict(b, seqs, [130, 1, 77, 301], w, sinks=20, recent=30)   # two stay as they are
    b.append(seqs, [3, 1, 2, ps])                               # onto the compacted pages
    run_attention(b, seqs, [3, 1, 2, 1], 4 * hkv)
    w = b.g.exponential(size=(4, 640)).astype(np.float32)
    evict(b, seqs, [5, 1, 0, 260], w)                           # no sinks, no recent; to nothing
    b.append(seqs, [0, 0, 4, 1])
    evict(b, [seqs[3]], [200], w[:1], sinks=3 * ps, recent=200 - 3 * ps) if 3 * ps <= 200 else None
    b.check()


def test_eviction_ties_signs_and_nan():
    b = Both(1, 1, 64, 16)
    s = b.new()
    b.append([s], [200])
    w = np.zeros((1, 200), dtype=np.float32)
    w[0, 50:60] = -0.0
    w[0, 70:75] = np.nan
    w[0, 80] = np.inf
    w[0, 81] = -np.inf
    w[0, 90:130] = 1.0
    w[0, 131] = 1e-45
    w[0, 132] = -1e-45
    evict(b, [s], [190], w, sinks=1, recent=1)
    w = np.concatenate([w[:, :0], np.full((1, 200), 3.0, dtype=np.float32)], 1)
    evict(b, [s], [150], w)                                      # all equal: the lowest stay
    w = np.full((1, 200), np.nan, dtype=np.float32)
    evict(b, [s], [20], w, recent=3)


def test_eviction_leaves_shared_pages_alone():
    b = Both(1, 2, 64, 16)
    s = b.new()
    b.append([s], [150])
    f, h = b.fork(s), b.fork(s)
    w = b.g.exponential(size=(2, 150)).astype(np.float32)
    evict(b, [f, h], [40, 90], w, sinks=33, recent=2)
    b.append([f, s], [20, 2])
    b.check()
    assert b.cache.page_table(f)[:2] == b.cache.page_table(s)[:2]   # two pages of sinks are still shared


def test_eviction_of_more_pages_than_one_launch_carries():
    b = Both(1, 1, 64, 8, pages=7000, seqs=70, max_pages=3600)
    s = b.new()
    b.append([s], [8 * 3500 + 3])
    many = [b.new() for _ in range(66)]
    b.append(many, [20] * 66)
    w = b.g.exponential(size=(67, 8 * 3500 + 3)).astype(np.float32)
    evict(b, [s] + many, [8 * 3200 + 1] + [9] * 66, w, sinks=9)


@pytest.mark.parametrize("n,keep", [(1023, 1000), (1024, 1), (1025, 1024), (5000, 2500), (33000, 4000)])
def test_selection_at_block_edges(n, keep):
    b = Both(1, 1, 64, 128, pages=-(-n // 128) * 2 + 2)
    s = b.new()
    b.append([s], [n])
    w = (b.g.integers(0, 50, size=(1, n)) / 7).astype(np.float32)    # many ties
    evict(b, [s], [keep], w)


def test_a_failed_eviction_changes_nothing():
    from paper_2609_04875_gb300 import binding
    b = Both(1, 2, 64, 16)
    s, t = b.new(), b.new()
    b.append([s, t], [150, 90])
    before = [b.cache.page_table(s), b.cache.page_table(t), b.cache.free_list(), b.cache.page_refs()]
    w = torch.rand((2, 150), device="cuda")
    w0 = w.clone()
    for k in range(3):
        b.cache.set_option("fail_launch_after", k)
        with pytest.raises(binding.PEError) as e:
            b.cache.evict_batch([s, t], [40, 50], w, sinks=1, recent=2)
        assert e.value.kind == "cuda"
        assert [b.cache.page_table(s), b.cache.page_table(t), b.cache.free_list(), b.cache.page_refs()] == before
        assert torch.equal(w, w0)
        b.check()
    b.cache.set_option("fail_launch_after", -1)
    evict(b, [s, t], [40, 50], w0.cpu().numpy(), sinks=1, recent=2)


def test_offsets_past_32_bits():
    """Pages at the end of pools of 4.5 GB of codes: append, read-back, attention on the codes and unpacked, weights,
    eviction, copy-on-write."""
    import paper_2609_04875_gb300 as pe
    pages = 34000
    b = Both(1, 8, 128, 128, pages=8, max_pages=16)
    b.cache = pe.PagedKVCache(1, 8, 128, 128, pages, 8, 16, init_free_order=list(range(pages))[::-1], kv_bits=8)
    s = b.new()
    b.append([s], [300])
    assert min(b.cache.page_table(s)) * 8 * 128 * 128 > 2 ** 32
    for n in (1, 5, 140):
        run_attention(b, [s], [n], 16)
    f = b.fork(s)
    b.append([f], [9])
    evict(b, [f], [200], b.g.exponential(size=(1, 309)).astype(np.float32), sinks=3)
    for q in (s, f):
        k, v = b.cache.read_kv(q)
        np.testing.assert_array_equal(to64(k), b.seqs[q].K)
        np.testing.assert_array_equal(to64(v), b.seqs[q].V)


# ---------------------------------------------------------------- refusals
def refused(kind, call, *args, **kw):
    from paper_2609_04875_gb300 import binding
    with pytest.raises(binding.PEError) as e:
        call(*args, **kw)
    assert e.value.kind == kind, e.value


def test_refusals():
    import paper_2609_04875_gb300 as pe
    b = Both(1, 2, 64, 16, pages=16)
    s, t = b.new(), b.new()
    b.append([s, t], [100, 60])
    c, q = b.cache, torch.zeros((1, 4, 64), device="cuda", dtype=torch.bfloat16)
    w = torch.zeros((1, 100), device="cuda")
    refused("range", c.replay_attn_weights_batch, [s], 0, q, [0, 1], w[:, :99].contiguous())
    refused("range", c.replay_attn_weights_batch, [s], 1, q, [0, 1], w)
    refused("invalid", c.replay_attn_weights_batch, [7], 0, q, [0, 1], w)
    with pytest.raises(TypeError):
        c.replay_attn_weights_batch([s], 0, q, [0, 1], w.double())
    with pytest.raises(TypeError):
        c.replay_attn_weights_batch([s], 0, q, [0, 1], w.cpu())
    with pytest.raises(ValueError):
        c.replay_attn_weights_batch([s], 0, q, [0, 1], torch.zeros((2, 100), device="cuda"))
    with pytest.raises(ValueError):
        c.replay_attn_weights_batch([s], 0, q, [0, 1], torch.zeros((100, 1), device="cuda").t()[:, ::2])
    with pytest.raises(ValueError):  # a view of longer rows: the columns count, not the stride
        c.replay_attn_weights_batch([s, t], 0, q.expand(2, 4, 64).contiguous(), [0, 1, 2], torch.zeros((2, 200), device="cuda")[:, :99])
    refused("range", c.read_kv_batch, [s], [90], [0, 11])
    refused("range", c.read_kv_batch, [s], [-1], [0, 1])
    refused("invalid", c.read_kv_batch, [5], [0], [0, 1])
    refused("invalid", c.read_kv_batch, [s, s], [0, 0], [0, 5, 3])
    w2 = torch.zeros((2, 100), device="cuda")
    refused("invalid", c.evict_batch, [s, s], [10, 10], w2)
    refused("invalid", c.evict_batch, [s], [10], w, sinks=6, recent=5)
    refused("invalid", c.evict_batch, [s], [-1], w)
    refused("invalid", c.evict_batch, [s], [10], w, sinks=-1)
    refused("range", c.evict_batch, [s], [10], w[:, :50].contiguous())
    refused("range", c.evict_batch, [s], [10], w, kept=torch.zeros((1, 9), device="cuda", dtype=torch.int32))
    refused("oom", c.evict_batch, [s, t], [90, 50], w2)     # 10 pages wanted, 5 free
    with pytest.raises(ValueError):
        c.evict_batch([s], [10], w, kept=torch.zeros((2, 9), device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        c.evict_batch([s], [10, 4], w)
    with pytest.raises(ValueError):
        pe.PagedKVCache(1, 2, 64, 16, 4, 1, 4, kv_bits=4)
    pool = torch.zeros((1, 4, 2, 16, 64), device="cuda", dtype=torch.bfloat16)
    with pytest.raises(pe.PEError) as e:
        pe.PagedKVCache(1, 2, 64, 16, 4, 1, 4, kv_bits=8, k_pool=pool, v_pool=pool.clone())
    assert e.value.kind == "invalid"
    b.check()
