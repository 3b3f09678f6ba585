"""Attention weights where scores are -infinity (bf16 caches: an 8-bit cache holds no infinity)."""
import math

import numpy as np
import pytest
import torch

import q8_model
from gpu_common import requires_cuda
from test_gpu_q8 import Both, bf16, to64, weights_bound

pytestmark = [pytest.mark.gpu, requires_cuda]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,where", [(1, range(0, 5)), (3, range(0, 140)), (2, [7, 128, 135, 299]), (40, range(100, 230))])
def test_weights_of_keys_whose_score_is_minus_infinity(n, where, d):
    """K of a bf16 cache may hold -infinity: such a key's weight is 0, wherever it stands, and the others' are as without it."""
    b = Both(1, 2, d, 16, bits=16)
    s = b.new()
    k, v = b.draw(300, 0.3), b.draw(300, 0.3)
    k[0, :, :, 3] = 0.5
    k[0, list(where), :, 3] = -np.inf
    b.append([s], [300], k, v)
    q, q64 = bf16(np.abs(b.g.standard_normal((n, 4, d))).astype(np.float32) + 0.1)   # (q > 0: a score is -inf, never NaN)
    w = torch.zeros((1, 300), device="cuda")
    b.cache.replay_attn_weights_batch([s], 0, q, [0, n], w)
    scale = 1 / math.sqrt(d)
    m = b.seqs[s]
    _, ref, _ = q8_model.attend(m.K[0], m.V[0], q64, scale)
    assert np.isfinite(ref).all() and (ref[list(where)] == 0).all()
    finite = np.where(np.isinf(m.K[0]), 0.0, m.K[0])
    assert (np.abs(to64(w[0]) - ref) <= weights_bound(finite, q64, scale, ref)).all()
    assert b.cache.device_status() == 0
