"""Calls on an 8-bit cache whose k-th device step fails (the "fail_launch_after" test hook: the step is not launched,
nothing faults), for every k: what the cache holds is then what it held before the call, bit for bit, values and scale
exponents, also on partly filled pages that an earlier step of the call had quantised again; so are an eviction's
weights."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import Both, bf16

pytestmark = [pytest.mark.gpu, requires_cuda]


def books(b):
    return ([b.cache.page_table(s) for s in b.seqs], [b.cache.seq_info(s) for s in b.seqs], b.cache.free_list(), b.cache.page_refs())


def fails_at_every_step(b, call, unchanged=lambda: None, at_least=2):
    """call() with its first step failing, then its second, .. until it succeeds; b's model stays at the state before."""
    from paper_2609_04875_gb300 import binding
    before = books(b)
    for k in range(100):
        b.cache.set_option("fail_launch_after", k)
        try:
            call()
        except binding.PEError as e:
            assert e.kind == "cuda" and "injected" in str(e), e
            assert books(b) == before, f"step {k}"
            b.check()
            unchanged()
            continue
        b.cache.set_option("fail_launch_after", -1)
        assert k >= at_least, f"the call had {k} steps that can fail"
        return
    raise AssertionError("the call never succeeded")


def larger(b, n):
    """Tokens whose scale leaves few of the kept values' bits."""
    return b.draw(n) * np.float32(2.0 ** 14)


def append_failing(b, seqs, counts):
    cu = np.concatenate([[0], np.cumsum(counts)]).tolist()
    (k, k64), (v, v64) = bf16(larger(b, cu[-1])), bf16(larger(b, cu[-1]))
    fails_at_every_step(b, lambda: b.cache.append_kv_batch(seqs, k, v, cu))
    for i, s in enumerate(seqs):
        b.seqs[s].append(k64[:, cu[i]: cu[i + 1]], v64[:, cu[i]: cu[i + 1]])
    b.check()


@pytest.mark.parametrize("L,hkv,d,ps", [(1, 1, 64, 8), (2, 3, 128, 16), (1, 2, 64, 128)])
def test_append_to_more_sequences_than_a_launch_carries(L, hkv, d, ps):
    b = Both(L, hkv, d, ps, pages=330, seqs=90)
    seqs = [b.new() for _ in range(75)]
    b.append(seqs, [1 + (5 * i) % (ps + 3) for i in range(75)])
    seqs += [b.fork(s) for s in seqs[:9]]          # shared pages: one of two holders copies, the other writes in place
    append_failing(b, seqs, [1 + (3 * i) % 4 for i in range(84)])


def test_append_of_more_pages_than_a_launch_carries():
    b = Both(1, 1, 64, 8, pages=3400, seqs=4, max_pages=3300)
    s, t = b.new(), b.new()
    b.append([s, t], [5, 11])
    append_failing(b, [t, s], [2, 8 * 3200])


def test_one_launch_has_nothing_to_undo():
    """A call of one step leaves nothing half done."""
    b = Both(1, 2, 64, 16)
    s = b.new()
    b.append([s], [21])
    (k, k64), (v, v64) = bf16(larger(b, 3)), bf16(larger(b, 3))
    fails_at_every_step(b, lambda: b.cache.append_kv(s, k, v), at_least=1)
    b.seqs[s].append(k64, v64)
    b.check()


@pytest.mark.parametrize("ps", [8, 64])
def test_rounds(ps):
    """Rounds append and attend in turn: a failure in any of them undoes the rounds before it too."""
    L, hkv, d, hq = 2, 2, 64, 4
    b = Both(L, hkv, d, ps, pages=90)
    s, t, e = b.new(), b.new(), b.new()
    b.append([s, t, e], [13, ps, 2 * ps + 3])      # part of a page, a whole one, part of one
    f = b.fork(s)                                  # its work begins in an earlier round than s's
    seqs, take = [s, t, e, f], np.array([[0, 1, 2, 1], [2, 0, 1, 3], [1, 3, 0, 0]], dtype=np.int32)
    n = take.sum(0)
    cu = np.concatenate([[0], np.cumsum(n)]).tolist()
    (k, k64), (v, v64) = bf16(larger(b, cu[-1])), bf16(larger(b, cu[-1]))
    q = bf16(b.g.standard_normal((L, cu[-1], hq, d)).astype(np.float32))[0]
    fails_at_every_step(b, lambda: b.cache.replay_rounds(seqs, take, cu, k, v, q), at_least=3)
    done = [0] * 4
    for row in take:
        for i, x in enumerate(seqs):
            at = slice(cu[i] + done[i], cu[i] + done[i] + int(row[i]))
            b.seqs[x].append(k64[:, at], v64[:, at])
            done[i] += int(row[i])
    b.check()
