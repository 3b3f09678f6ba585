"""An eviction of more sequences, or pages, than one launch carries, whose k-th device step fails, for every k: cache and
weights are then as before the call, so that the same call again keeps what it would have kept."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import Both, evict
from test_gpu_q8_failures import fails_at_every_step

pytestmark = [pytest.mark.gpu, requires_cuda]


@pytest.mark.parametrize("bits", [8, 16])
@pytest.mark.parametrize("n,longest", [(65, 40), (140, 40), (3, 8 * 3200)])
def test_an_eviction_of_several_launches(n, longest, bits):
    ps = 8
    b = Both(1, 2, 64, ps, pages=3 * (longest // ps + 1) + 14 * n + 3300, seqs=n, bits=bits, max_pages=longest // ps + 8)
    seqs = [b.new() for _ in range(n)]
    lens = [longest] + [9 + (7 * i) % 31 for i in range(n - 1)]
    b.append(seqs, lens)
    keep = [longest - 5] + [min(x, 8 + i % 5) for i, x in enumerate(lens[1:])]   # some stay as they are
    first = b.g.exponential(size=(n, longest)).astype(np.float32)
    w = torch.from_numpy(first).cuda()

    def unchanged():
        assert torch.equal(w.cpu(), torch.from_numpy(first))

    result = {}

    def call():
        result["kept"] = b.cache.evict_batch(seqs, keep, w, sinks=2, recent=3)

    fails_at_every_step(b, call, unchanged, at_least=4)
    for i, s in enumerate(seqs):
        want, left = b.seqs[s].evict(keep[i], first[i], 2, 3)
        np.testing.assert_array_equal(result["kept"][i, : len(want)].cpu().numpy(), want)
        np.testing.assert_array_equal(w[i].cpu().numpy(), left)
    b.check()
    evict(b, seqs, [min(x, 7) for x in keep], b.g.exponential(size=(n, longest)).astype(np.float32), sinks=1)
