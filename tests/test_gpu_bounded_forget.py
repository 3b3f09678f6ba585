"""What a forget request leaves of the forgotten turns in a bounded session's account: nothing, so that later evictions
are those of a session that never saw them (the crop on a page's end, where the kept codes have no trace of them either)."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import bf16

pytestmark = [pytest.mark.gpu, requires_cuda]

L, HQ, HKV, D, PS = 2, 4, 2, 64, 16


def agents(n):
    from paper_2609_04875_gb300.bounded import BoundedAgents
    return BoundedAgents(n, L, HQ, HKV, D, budget=80, slack=16, sinks=3, recent=8, page_size=PS)


def tokens(g, n):
    return [bf16(g.standard_normal((L, n, h, D)).astype(np.float32))[0] for h in (HKV, HKV, HQ)]


def side_by_side(*parts):
    return [torch.cat(x, 1).contiguous() for x in zip(*parts)]


def test_later_evictions_do_not_depend_on_forgotten_turns():
    g = np.random.default_rng(7)
    prompt, one, other = tokens(g, 64), tokens(g, 20), tokens(g, 20)
    other[2] *= 6                                   # queries that draw on few keys
    b = agents(3)
    b.append(*side_by_side(prompt, prompt, prompt), [64, 64, 64])
    b.append(*side_by_side(one, other), [20, 20, 0])
    assert b.forget(0, 65) == 64 and b.forget(1, 65) == 64 and b.forget(2, 65) == 64
    assert torch.equal(b.weights, torch.zeros_like(b.weights))
    while b.lengths()[0] != 80:                     # on to the first eviction
        step = tokens(g, 3)
        b.append(*side_by_side(step, step, step), [3, 3, 3])
    assert b.lengths() == [80, 80, 80]
    for i in (1, 2):
        assert torch.equal(b.origin[0], b.origin[i])
        assert torch.equal(b.weights[0], b.weights[i])


def test_the_kept_queries_counted_again():
    g = np.random.default_rng(8)
    prompt, more = tokens(g, 64), tokens(g, 20)
    b = agents(2)
    b.append(*side_by_side(prompt, prompt), [64, 64])
    b.append(*more, [20, 0])
    assert b.forget(0, 65) == 64
    b.recount(0, prompt[2])
    assert float(b.weights[1].sum()) > 0
    assert torch.equal(b.weights[0], b.weights[1])  # the same call on the same values
    assert b.forget(0, 1) == 0
    b.recount(0, prompt[2][:, :0].contiguous())
    assert float(b.weights[0].abs().sum()) == 0
    for wrong in (prompt[2][:, :63], prompt[2][:1], prompt[0]):
        with pytest.raises(ValueError):
            b.recount(1, wrong.contiguous())
    assert b.cache.device_status() == 0
