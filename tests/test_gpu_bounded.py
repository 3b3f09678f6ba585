"""The bounded-session driver against the 8-bit cache's definition in 64 bits: prompts, steps with evictions, a forget
request in a session that has lost tokens."""
import numpy as np
import pytest
import torch

import q8_model
from gpu_common import requires_cuda
from test_gpu_q8 import assert_attention, bf16, to64

pytestmark = [pytest.mark.gpu, requires_cuda]


def test_steps_evictions_and_a_forget_request():
    from paper_2609_04875_gb300.bounded import BoundedAgents
    agents, L, hq, hkv, d, ps = 3, 2, 4, 2, 64, 16
    b = BoundedAgents(agents, L, hq, hkv, d, budget=40, slack=6, sinks=3, recent=8, page_size=ps, longest_prompt=70)
    model = [q8_model.Seq(L, hkv, d, ps) for _ in range(agents)]
    origin = [np.zeros(0, dtype=int) for _ in range(agents)]
    seen = [0] * agents
    g = np.random.default_rng(5)

    def step(counts):
        cu = np.concatenate([[0], np.cumsum(counts)])
        draw = lambda h: bf16(g.standard_normal((L, cu[-1], h, d)).astype(np.float32))  # noqa: E731
        (k, k64), (v, v64), (q, q64) = draw(hkv), draw(hkv), draw(hq)
        before = b.weights.clone()
        out = b.append(k, v, q, counts)
        for i, n in enumerate(counts):
            at = slice(cu[i], cu[i + 1])
            model[i].append(k64[:, at], v64[:, at])
            origin[i] = np.concatenate([origin[i], seen[i] + np.arange(n)])
            seen[i] += n
            if n == 0:
                continue
            w = to64(before[i])
            for layer in range(L):
                w[: len(model[i])] += assert_attention(out[layer, at], model[i], q64[layer, at], 1 / np.sqrt(d), layer, f"agent {i}")
            if len(model[i]) > 46:
                # the driver selects by its own account: close to w, and its choice is what the model follows
                kept = b.origin[i, :40].cpu().numpy()
                rows = np.searchsorted(origin[i], kept)
                assert np.array_equal(origin[i][rows], kept) and (np.diff(kept) > 0).all()
                T = len(model[i])
                assert np.array_equal(rows[:3], np.arange(3)) and np.array_equal(rows[-8:], np.arange(T - 8, T))
                lost = np.setdiff1d(np.arange(T), rows)
                assert w[rows[3:-8]].min() >= w[lost].max() - 1e-4
                model[i].K, model[i].V, model[i].E = model[i].K[:, rows], model[i].V[:, rows], model[i].E[:, :0]
                model[i]._hold(0)
                origin[i] = kept
                w = np.concatenate([w[rows], np.zeros(b.columns - 40)])
            np.testing.assert_allclose(to64(b.weights[i]), w, atol=1e-4)
        assert b.lengths() == [len(m) for m in model]
        for i, m in enumerate(model):
            if len(m):
                kk, vv = b.cache.read_kv(b.seqs[i])
                np.testing.assert_array_equal(to64(kk), m.K)
                np.testing.assert_array_equal(to64(vv), m.V)

    step([70, 5, 46])
    assert b.lengths() == [40, 5, 46]
    for _ in range(9):
        step([1, 1, 1])
    step([0, 3, 2])
    tau = int(origin[0][20]) + 1                      # the 21st held token's position in the whole session
    assert b.forget(0, tau) == 20
    model[0].crop(21)
    origin[0], seen[0] = origin[0][:20], tau - 1
    step([4, 1, 1])
    with pytest.raises(ValueError):
        b.forget(1, 1000)
    with pytest.raises(ValueError):
        BoundedAgents(1, 1, 1, 1, 64, budget=10, sinks=5, recent=6)
    assert b.cache.device_status() == 0
