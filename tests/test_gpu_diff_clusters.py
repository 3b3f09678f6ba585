"""Differential attention of few rows on few keys by clusters of CTAs, a unit each: no more of them than the device holds at
once."""
import pytest
import torch

from test_gpu_diff import Setup
from test_gpu_rope import cu_of

pytestmark = pytest.mark.gpu
pe = pytest.importorskip("paper_2609_04875_gb300")


# sequences, keys, and the launches: one of whole units, or one that cuts them and a merge.  (152 SMs hold 15 clusters of 8 CTAs
# and 36 of 4.)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("B,T,launches", [(15, 2000, 1), (16, 2000, 2), (19, 2000, 2), (16, 1000, 1), (36, 1000, 1), (37, 1000, 2), (38, 600, 1),
                                          (64, 200, 1)])
def test_units_that_do_not_fit_at_once_are_cut(B, T, launches, d):
    lens = [T - (i * 5) % 40 for i in range(B)]
    s = Setup(lens, 2, d, 16, seed=B + T)
    q, lam, gain = s.inputs([1] * B, 8)
    cu = cu_of([1] * B)
    before = s.cache.kernel_launches()
    out = s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=gain)
    assert s.cache.kernel_launches() - before == launches
    s.check(out, s.seqs, q, cu, lam, gain)
    assert torch.equal(out, s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=gain))


def test_asked_first_in_a_capture():
    """The device is asked what it holds at a cache's first call, which may be one that is captured."""
    s = Setup([700, 300], 4, 64, 16, seed=1)
    q, lam, gain = s.inputs([1, 2], 8)
    cu = [0, 1, 3]
    out = torch.empty((3, 4, 128), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.diff_attn_batch(s.seqs, 0, q, cu, lam, gain=gain, out=out)
    graph.replay()
    torch.cuda.synchronize()
    s.check(out, s.seqs, q, cu, lam, gain)
