"""Differential attention over the paged cache, against 64 bits."""
import math

import pytest
import torch

import rope_diff_model as model
from test_gpu_rope import cu_of, freqs, gen, randn

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")


class Setup:
    """Sequences of `lens` tokens on shuffled pages; K and V with columns of unequal size and some large tokens."""

    def __init__(self, lens, hkv, d, ps, seed=0, bits=16, L=1, outliers=0.01, slack=3, **kw):
        g = self.g = gen(seed)
        self.lens, self.hkv, self.d, self.L = lens, hkv, d, L
        pages = sum(-(-t // ps) for t in lens) + slack
        order = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).tolist()
        self.cache = pe.PagedKVCache(L, hkv, d, ps, pages, len(lens) + 1, max(-(-t // ps) for t in lens) + 1, init_free_order=order,
                                     kv_bits=bits, **kw)
        self.seqs = [self.cache.seq_create() for _ in lens]
        N = sum(lens)
        big = 1 + 7 * (torch.rand((1, N, 1, 1), generator=g, device="cuda") < outliers).float()
        col = torch.exp(0.5 * torch.randn((1, 1, hkv, d), generator=g, device="cuda"))
        self.K, self.V = [(torch.randn((L, N, hkv, d), generator=g, device="cuda") * big * col).to(torch.bfloat16) for _ in range(2)]
        self.cache.append_kv_batch(self.seqs, self.K, self.V, cu_of(lens))

    def inputs(self, counts, hq, norm=True):
        q = randn(self.g, sum(counts), hq, self.d)
        lam = 0.5 + 0.15 * torch.randn(hq // 2, generator=self.g, device="cuda")
        gain = 0.4 * (1 + 0.1 * torch.randn(2 * self.d, generator=self.g, device="cuda")) if norm else None
        return q, lam, gain

    def check(self, out, seqs, q, cu, lam, gain, layer=0, scale=None, eps=1e-5, what=""):
        scale = 1.0 / math.sqrt(self.d) if scale is None else scale
        for i, s in enumerate(seqs):
            a, b = cu[i], cu[i + 1]
            if a == b:
                continue
            k, v = self.cache.read_kv(s)
            want, bound = model.diff_attention(q[a:b].double(), k[layer].double(), v[layer].double(), lam.double(),
                                               None if gain is None else gain.double(), eps, scale, q.shape[1] // self.hkv)
            model.check_diff(out[a:b], want, bound, f"{what} sequence {i}")


# lens, counts, hq, hkv, d, ps, norm
CASES = [
    ([640], [1], 8, 8, 64, 16, True),
    ([1], [1], 2, 2, 128, 16, True),
    ([1, 2, 63, 64, 65, 127, 128, 129], [1] * 8, 8, 2, 64, 8, True),
    ([700, 33, 401], [1, 1, 1], 32, 8, 128, 16, True),
    ([3000], [1], 16, 2, 128, 64, False),
    ([515, 5, 200], [16, 5, 0], 32, 8, 128, 16, False),
    ([300, 300], [15, 300], 8, 4, 64, 32, True),
    ([257], [257], 4, 2, 128, 128, True),
    ([1000], [70], 64, 4, 64, 16, True),
    ([260, 90], [65, 33], 4, 4, 128, 8, True),
    ([900, 1100], [200, 130], 16, 4, 128, 16, True),
    ([400], [3], 256, 2, 64, 32, False),
    ([2000, 70, 1500], [700, 70, 1], 8, 2, 64, 16, True),
    ([5000], [900], 32, 8, 128, 16, True),
]


@pytest.mark.parametrize("lens,counts,hq,hkv,d,ps,norm", CASES)
def test_against_64_bits(lens, counts, hq, hkv, d, ps, norm):
    s = Setup(lens, hkv, d, ps, seed=sum(lens) + hq)
    q, lam, gain = s.inputs(counts, hq, norm)
    cu = cu_of(counts)
    out = s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=gain)
    assert out.shape == (sum(counts), hq // 2, 2 * d) and out.dtype == torch.bfloat16
    s.check(out, s.seqs, q, cu, lam, gain)
    assert torch.equal(out, s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=gain))
    assert s.cache.device_status() == 0


@pytest.mark.parametrize("counts", [[1, 1], [40, 7], [150, 300]])
@pytest.mark.parametrize("d", [64, 128])
def test_8_bit_caches_and_layers(d, counts):
    s = Setup([600, 333], 4, d, 16, seed=d, bits=8, L=3)
    q, lam, gain = s.inputs(counts, 8)
    for layer in (2, 0):
        out = s.cache.diff_attn_batch(s.seqs, layer, q, cu_of(counts), lam, gain=gain)
        s.check(out, s.seqs, q, cu_of(counts), lam, gain, layer=layer)


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("std", [0.01, 8.0, 30.0])
def test_flat_and_peaked_scores(std, n):
    s = Setup([1500], 4, 128, 16, seed=int(std * 100) + n, outliers=0.0)
    q, lam, gain = s.inputs([n], 8)
    q = (q.float() * std).to(torch.bfloat16)
    out = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    s.check(out, s.seqs, q, [0, n], lam, gain, what=f"std {std}")


@pytest.mark.parametrize("n", [1, 130])
@pytest.mark.parametrize("at", [64, 100, 700, 1300])
def test_references_that_move(at, n):
    """Scores that jump by hundreds at a key, in one map alone and in some queries only."""
    s = Setup([1500], 2, 128, 16, seed=at + n, outliers=0.0)
    q, lam, _ = s.inputs([n], 4, False)
    K = s.K.clone()
    K[:, at:, 0] = (K[:, at:, 0].float() * 40).to(torch.bfloat16)
    s.cache.crop(s.seqs[0], 1)
    s.cache.append_kv(s.seqs[0], K, s.V)
    q[::3, 2] *= 4
    out = s.cache.diff_attn(s.seqs[0], 0, q, lam)
    s.check(out, s.seqs, q, [0, n], lam, None)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [5, 100, 400])
def test_what_a_row_does_not_see_does_not_reach_it(n, d):
    """NaN and infinities in K and V of the last positions: rows before them are as without, rows that see them are not
    finite.  And what a crop left behind in the last page's slots reaches no row."""
    s = Setup([600], 4, d, 32, seed=n + d)
    q, lam, gain = s.inputs([n], 8)
    seq, twin = s.seqs[0], s.cache.seq_fork(s.seqs[0])
    want = s.cache.diff_attn(seq, 0, q, lam, gain=gain)
    s.cache.seq_release(twin)
    bad_k, bad_v = s.K.clone(), s.V.clone()
    bad_v[0, 598, 1, 3], bad_v[0, 597, 0, :], bad_k[0, 599, 2, 0] = float("nan"), float("inf"), float("nan")
    s.cache.crop(seq, 1)
    s.cache.append_kv(seq, bad_k, bad_v)
    got = s.cache.diff_attn(seq, 0, q, lam, gain=gain)
    # head i reads kv-heads 2j, 2j + 1 with j = i // 2: V of j = 0 is bad from 597 on, K of j = 1 at 599
    assert torch.equal(got[: n - 3], want[: n - 3])
    assert torch.equal(got[: n - 1, 2:], want[: n - 1, 2:])
    assert not torch.isfinite(got[n - 3:, :2]).all(dim=2).any() and torch.isnan(got[n - 1, 2:]).all()
    s.cache.crop(seq, 598)  # 597 tokens, the bad ones in the slots behind them
    m = min(n, 300)
    got = s.cache.diff_attn(seq, 0, q[:m], lam, gain=gain)
    s.check(got, s.seqs, q[:m], [0, m], lam, gain)
    assert torch.isfinite(got).all()


def test_scores_of_minus_infinity():
    """Keys whose score is -infinity draw nothing; a map that sees no others counts as zero."""
    for n in (1, 90):
        s = Setup([200], 2, 64, 16, seed=n, outliers=0.0)
        q, lam, _ = s.inputs([n], 4, False)
        q = (q.float().abs() + 0.1).to(torch.bfloat16)
        K, ninf = s.K.clone(), float("-inf")
        K[0, :64, 0], K[0, 70:, 0, 5] = ninf, ninf
        s.cache.crop(s.seqs[0], 1)
        s.cache.append_kv(s.seqs[0], K, s.V)
        out = s.cache.diff_attn(s.seqs[0], 0, q, lam)
        s.check(out, s.seqs, q, [0, n], lam, None, what=f"some, n {n}")
        K[0, :, 1, 7] = ninf
        s.cache.crop(s.seqs[0], 1)
        s.cache.append_kv(s.seqs[0], K, s.V)
        zero = s.cache.diff_attn(s.seqs[0], 0, q, lam)
        one = s.cache.diff_attn(s.seqs[0], 0, q, torch.zeros_like(lam))
        assert torch.equal(zero, one) and torch.isfinite(zero).all()


def test_same_sequence_twice_and_a_fork():
    s = Setup([500], 4, 64, 16, seed=3)
    f = s.cache.seq_fork(s.seqs[0])
    seqs, counts = [s.seqs[0], f, s.seqs[0]], [3, 3, 90]
    q, lam, gain = s.inputs(counts, 8)
    q[3:6] = q[:3]
    out = s.cache.diff_attn_batch(seqs, 0, q, cu_of(counts), lam, gain=gain)
    s.check(out, seqs, q, cu_of(counts), lam, gain)
    assert torch.equal(out[:3], out[3:6])


def test_more_sequences_than_a_launch_takes():
    lens = [1 + (i * 37) % 300 for i in range(70)]
    s = Setup(lens, 2, 64, 16, seed=4)
    counts = [min(t, 1 + (i * 13) % 50) for i, t in enumerate(lens)]
    q, lam, gain = s.inputs(counts, 4)
    out = s.cache.diff_attn_batch(s.seqs, 0, q, cu_of(counts), lam, gain=gain)
    s.check(out, s.seqs, q, cu_of(counts), lam, gain)


@pytest.mark.parametrize("mib", [2, 9])
def test_small_workspaces(mib):
    """Launches of as many rows as their partials fit."""
    s = Setup([900, 1300], 4, 128, 16, seed=mib, workspace_bytes=mib << 20)
    for counts in ([1, 1], [20, 3], [300, 500]):
        q, lam, gain = s.inputs(counts, 8)
        out = s.cache.diff_attn_batch(s.seqs, 0, q, cu_of(counts), lam, gain=gain)
        s.check(out, s.seqs, q, cu_of(counts), lam, gain, what=str(counts))


def test_debug_poison_and_rows_behind():
    s = Setup([300], 2, 64, 16, seed=5)
    s.cache.set_option("debug_poison", 1)
    s.cache.crop(s.seqs[0], 251)
    q, lam, gain = s.inputs([40], 4)
    base = torch.full((60, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    wide = torch.full((131,), 3.0, device="cuda")  # lambda and gain where a vector load may not begin
    wide[1:129], lam2 = gain, torch.cat([lam[:1], lam])[1:]
    out = s.cache.diff_attn(s.seqs[0], 0, q, lam2, gain=wide[1:129], out=base[10:50])
    s.check(out, s.seqs, q, [0, 40], lam, gain)
    assert (base[:10] == 7).all() and (base[50:] == 7).all()


def test_offsets_past_32_bits():
    free, _ = torch.cuda.mem_get_info()
    if free < 40 << 30:
        pytest.skip("needs 40 GB")
    g = gen(6)
    pages = (1 << 32) // (2 * 16 * 128) + 64
    cache = pe.PagedKVCache(1, 2, 128, 16, pages, 1, 64, init_free_order=list(range(pages))[::-1])
    seq = cache.seq_create()
    K, V = randn(g, 1, 700, 2, 128), randn(g, 1, 700, 2, 128)
    cache.append_kv(seq, K, V)
    lam = torch.tensor([0.4, 0.6], device="cuda")
    for n in (1, 300):
        q = randn(g, n, 4, 128)
        out = cache.diff_attn(seq, 0, q, lam)
        want, bound = model.diff_attention(q.double(), K[0].double(), V[0].double(), lam.double(), None, 1e-5, 128 ** -0.5, 2)
        model.check_diff(out, want, bound, f"n {n}")


@pytest.mark.parametrize("n", [1, 260])
def test_streams_and_graphs(n):
    s = Setup([900], 4, 128, 16, seed=7)
    q, lam, gain = s.inputs([n], 8)
    want = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    # two graphs that share the cache's workspace, replayed in turn on other contents
    graphs, outs, xs = [], [], []
    for _ in range(2):
        x, out = q.clone(), torch.empty_like(want)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.cache.diff_attn(s.seqs[0], 0, x, lam, gain=gain, out=out)
        graphs.append(graph)
        outs.append(out)
        xs.append(x)
    xs[1].copy_(q.flip(0) * 0.5)
    for _ in range(3):
        for graph in graphs:
            graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want)
    s.check(outs[1], s.seqs, xs[1], [0, n], lam, gain)


@pytest.mark.parametrize("bits", [16, 8])
def test_a_step_as_a_model_makes_it(bits):
    """Crop, append with the rotation, differential attention of the same tokens' rotated queries, layer by layer; then a
    token more."""
    L, hq, hkv, d, lens = 2, 8, 4, 64, [210, 77]
    s = Setup(lens, hkv, d, 16, seed=8, bits=bits, L=L, slack=20)
    rope = pe.Rope(freqs(32))
    s.cache.crop_batch(s.seqs, [151, 41])
    for counts in ([60, 30], [1, 1]):
        cu = cu_of(counts)
        K, V, Q = [randn(s.g, L, cu[-1], h, d) for h in (hkv, hkv, hq)]
        _, lam, gain = s.inputs([1], hq)
        before = [s.cache.seq_info(x)[0] for x in s.seqs]
        rq = s.cache.append_kv_rope_batch(s.seqs, K, V, cu, rope, Q=Q)
        pos = torch.tensor([[t + j for t, n in zip(before, counts) for j in range(n)]], device="cuda", dtype=torch.int32)
        model.check_rotated(rq, *model.rotated(Q, pos, freqs(32)))
        for layer in range(L):
            out = s.cache.diff_attn_batch(s.seqs, layer, rq[layer], cu, lam, gain=gain, eps=1e-6)
            s.check(out, s.seqs, rq[layer], cu, lam, gain, layer=layer, eps=1e-6)
            # the cache's own attention reads the same keys
            s.cache.replay_attn_batch(s.seqs, layer, rq[layer], cu)


def test_prepared_calls_are_the_plain_ones():
    s = Setup([300, 90], 4, 64, 16, seed=11, slack=20)
    q, lam, gain = s.inputs([2, 2], 8)
    cu, rope = [0, 2, 4], pe.Rope(freqs(32))
    K, V = randn(s.g, 1, 4, 4, 64), randn(s.g, 1, 4, 4, 64)
    rq, out, x = torch.empty_like(q)[None], torch.empty((4, 4, 128), dtype=torch.bfloat16, device="cuda"), torch.empty_like(q)
    append = s.cache.prepare_append_kv_rope_batch(s.seqs, K, V, cu, rope, Q=q[None], Q_out=rq)
    rotate = s.cache.prepare_rotate_batch(s.seqs, q, cu, rope, x)
    attend = s.cache.prepare_diff_attn_batch(s.seqs, 0, rq[0], cu, lam, out, gain=gain)
    for _ in range(2):
        append()
        rotate()
        attend()
        assert torch.equal(x, rq[0]) and torch.equal(x, s.cache.rotate_batch(s.seqs, q, cu, rope))
        assert torch.equal(out, s.cache.diff_attn_batch(s.seqs, 0, rq[0], cu, lam, gain=gain))
    assert [s.cache.seq_info(i)[0] for i in s.seqs] == [304, 94]
    s.check(out, s.seqs, rq[0], cu, lam, gain)
    for call, args, kw in [(s.cache.prepare_append_kv_rope_batch, (s.seqs, K, V, cu, rope), {"Q": q[None]}),
                           (s.cache.prepare_rotate_batch, (s.seqs, q, cu, rope, x[:3]), {}),
                           (s.cache.prepare_rotate_batch, (s.seqs, q, cu, rope, x), {"positions": torch.zeros((2, 4), dtype=torch.int32, device="cuda")}),
                           (s.cache.prepare_diff_attn_batch, (s.seqs, 0, q, cu, lam, x), {})]:
        with pytest.raises(ValueError):
            call(*args, **kw)


def test_a_failed_launch():
    s = Setup([600], 4, 64, 16, seed=9)
    q, lam, gain = s.inputs([80], 8)
    want = s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    s.cache.set_option("fail_launch_after", 0)
    with pytest.raises(pe.PEError, match="injected"):
        s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain)
    assert torch.equal(s.cache.diff_attn(s.seqs[0], 0, q, lam, gain=gain), want)


def test_refusals():
    s = Setup([50, 60], 2, 64, 16, seed=10)
    q, lam, gain = s.inputs([4, 4], 4)
    seqs, cu = s.seqs, [0, 4, 8]
    call = s.cache.diff_attn_batch
    for args, kw, err in [
        ((seqs, 0, q, cu, lam.double()), {}, TypeError), ((seqs, 0, q, cu, lam[:1]), {}, ValueError),
        ((seqs, 0, q, cu, lam.cpu()), {}, TypeError), ((seqs, 0, q, cu, lam.repeat(2)[::2]), {}, ValueError),
        ((seqs, 0, q, cu, lam), {"gain": gain[:64]}, ValueError), ((seqs, 0, q, cu, lam), {"eps": -1.0}, pe.PEError),
        ((seqs, 0, q, cu, lam), {"eps": float("nan")}, pe.PEError), ((seqs, 0, q, [0, 4], lam), {}, ValueError),
        ((seqs, 0, q.float(), cu, lam), {}, TypeError), ((seqs, 0, q[:, :3], cu, lam), {}, ValueError),
        ((seqs, 5, q, cu, lam), {}, pe.PEError), ((seqs, 0, q, cu, lam), {"softmax_scale": 0.0}, pe.PEError),
        (([seqs[0], 7], 0, q, cu, lam), {}, pe.PEError), ((seqs, 0, q, cu, lam), {"out": torch.empty_like(q)}, ValueError),
        ((seqs, 0, q, cu, lam), {"out": q.view(8, 2, 128)}, pe.PEError),
        ((seqs, 0, torch.cat([q] * 8), [0, 51, 64], lam), {}, pe.PEError),
    ]:
        with pytest.raises(err):
            call(*args, **kw)
    odd = pe.PagedKVCache(1, 3, 64, 16, 8, 1, 8)
    x = odd.seq_create()
    odd.append_kv(x, randn(s.g, 1, 5, 3, 64), randn(s.g, 1, 5, 3, 64))
    with pytest.raises(pe.PEError, match="pairs of kv-heads"):
        odd.diff_attn(x, 0, randn(s.g, 1, 6, 64), torch.zeros(3, device="cuda"))
    host = pe.PagedKVCache(1, 2, 64, 16, 8, 1, 8, host_only=True)
    with pytest.raises(ValueError):
        host.diff_attn_batch([host.seq_create()], 0, q, [0, 8], lam)
    tiny = pe.PagedKVCache(1, 2, 64, 16, 8, 1, 8, workspace_bytes=1024)
    y = tiny.seq_create()
    tiny.append_kv(y, randn(s.g, 1, 5, 2, 64), randn(s.g, 1, 5, 2, 64))
    for n in (1, 5):
        with pytest.raises(pe.PEError, match="workspace"):
            tiny.diff_attn(y, 0, randn(s.g, n, 2 if n == 1 else 64, 64), torch.zeros(1 if n == 1 else 32, device="cuda"))
    none = s.cache.diff_attn_batch(seqs, 0, q[:0], [0, 0, 0], lam)
    assert none.shape == (0, 2, 128)
