"""What a crop leaves of the tokens it removed from an 8-bit cache: where it ends on a page's end, nothing; inside a page,
the scale that the removed tokens set, to which the kept tokens of that page stay rounded."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import Both, bf16, to64

pytestmark = [pytest.mark.gpu, requires_cuda]


@pytest.mark.parametrize("size", [6, 10, 20])
def test_on_a_pages_end_a_crop_leaves_no_trace(size):
    b = Both(2, 2, 64, 16)
    s, fresh = b.new(), b.new()
    k, v = b.draw(70), b.draw(70)
    b.append([fresh], [70], k, v)
    b.append([s], [48], k[:, :48], v[:, :48])
    b.append([s], [30], b.draw(30) * np.float32(2.0 ** size), b.draw(30) * np.float32(2.0 ** size))
    b.crop(s, 49)
    b.append([s], [22], k[:, 48:], v[:, 48:])
    b.check()
    np.testing.assert_array_equal(b.seqs[s].K, b.seqs[fresh].K)
    np.testing.assert_array_equal(b.seqs[s].V, b.seqs[fresh].V)
    np.testing.assert_array_equal(b.seqs[s].E, b.seqs[fresh].E)
    q = bf16(np.random.default_rng(3).standard_normal((22, 4, 64)).astype(np.float32))[0]
    for layer in range(2):
        assert torch.equal(b.cache.replay_attn(s, layer, q), b.cache.replay_attn(fresh, layer, q))


@pytest.mark.parametrize("size,off", [(6, 1e-3), (10, 1e-2), (14, 0.2), (20, 0.5)])
def test_inside_a_page_the_removed_tokens_scale_stays(size, off):
    """What is held is pinned: the page's values with the removed tokens' exponents, which the replay's do not raise; at
    least `off` of them differ from a fresh session's."""
    b = Both(2, 2, 128, 16)
    s, fresh = b.new(), b.new()
    k, v = b.draw(40, 0.0), b.draw(40, 0.0)
    b.append([fresh], [40], k, v)
    b.append([s], [40], k, v)
    b.append([s], [8], b.draw(8, 0.0) * np.float32(2.0 ** size), b.draw(8, 0.0) * np.float32(2.0 ** size))
    b.crop(s, 41)
    b.check()
    page = slice(32, 40)
    for got, clean in ((b.seqs[s].K, b.seqs[fresh].K), (b.seqs[s].V, b.seqs[fresh].V)):
        np.testing.assert_array_equal(got[:, :32], clean[:, :32])
        differ = np.mean(got[:, page] != clean[:, page])
        assert differ >= off
    # the way without a trace: the crop goes back to the page's start, and its kept tokens are given again
    b.crop(s, 33)
    b.append([s], [8], k[:, 32:], v[:, 32:])
    b.check()
    np.testing.assert_array_equal(b.seqs[s].K, b.seqs[fresh].K)
    np.testing.assert_array_equal(b.seqs[s].V, b.seqs[fresh].V)
