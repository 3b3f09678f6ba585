"""Bounded sessions whose keys and queries turn by their positions in the whole sessions: after evictions and a forget request
the held keys are those that stood there, rotated by where they stood, and queries attend them rotated by theirs."""
import numpy as np
import pytest
import torch

import rope_diff_model as model
from gpu_common import requires_cuda

pytestmark = [pytest.mark.gpu, requires_cuda]


@pytest.mark.parametrize("axes", [None, [i % 3 for i in range(32)]])
def test_rotation_follows_the_whole_session(axes):
    import paper_2609_04875_gb300 as pe
    from paper_2609_04875_gb300.bounded import BoundedAgents
    agents, L, hq, hkv, d = 2, 2, 4, 2, 64
    freq = [10000.0 ** (-i / 32) for i in range(32)]
    b = BoundedAgents(agents, L, hq, hkv, d, budget=40, slack=6, sinks=3, recent=8, longest_prompt=70, rope=pe.Rope(freq, axis=axes))
    n_axes = 1 if axes is None else 3
    g = torch.Generator("cuda").manual_seed(3)
    keys = [[] for _ in range(agents)]  # of the whole sessions, rotated, in 64 bits

    def rotated(x, positions):
        pos = torch.tensor(positions, device="cuda")[None].expand(n_axes, -1)
        return model.rotated(x, pos, freq, axes)[0]

    def step(counts):
        N = sum(counts)
        K, V, Q = [torch.randn((L, N, h, d), generator=g, device="cuda").to(torch.bfloat16) for h in (hkv, hkv, hq)]
        first, lens, at = list(b.seen), b.lengths(), 0
        out = b.append(K, V, Q, counts)
        for i, n in enumerate(counts):
            own = list(range(first[i], first[i] + n))
            k = rotated(K[:, at:at + n], own)
            keys[i] += [k[:, j] for j in range(n)]
            q = rotated(Q[:, at:at + n], own).to(torch.bfloat16).double()
            held = b.lengths()[i]
            kk, vv = [x.double() for x in b.cache.read_kv(b.seqs[i])]
            origin = b.origin[i, :held].tolist()
            want = torch.stack([keys[i][j] for j in origin], dim=1)
            # three roundings to e4m3 at most (an append, and an eviction's or two), steps of a page's scale at least
            off = (kk - want).abs() - 3 * torch.maximum(model.E8 * want.abs(), want.abs().amax() / 448 * 2 * 2.0 ** -10)
            assert off.max().item() <= 0, (i, off.max().item())
            if held == lens[i] + n and n:  # nothing was evicted: the outputs are these keys' attention
                for layer in range(L):
                    for h in range(hq):
                        s = q[layer, :, h] @ kk[layer, :, h // 2].t() * d ** -0.5
                        seen = torch.arange(held, device="cuda")[None] <= torch.arange(held - n, held, device="cuda")[:, None]
                        w = torch.softmax(s.masked_fill(~seen, -np.inf), dim=1)
                        v = vv[layer, :, h // 2]
                        bound = 4 * model.EB * (w @ v.abs()) + 1e-6
                        assert ((out[layer, at:at + n, h].double() - w @ v).abs() - bound).max().item() <= 0
            at += n

    step([70, 5])
    assert b.lengths() == [40, 5]
    for _ in range(9):
        step([1, 1])
    step([0, 3])
    tau = b.origin[0, 20].item() + 1
    assert b.forget(0, tau) == 20
    del keys[0][tau - 1:]
    step([4, 1])
    held = b.lengths()[0]
    Q = torch.randn((L, held, hq, d), generator=g, device="cuda").to(torch.bfloat16)
    b.recount(0, Q)
    # every query's weights add up to one, layer by layer and head by head
    assert abs(b.weights[0].sum().item() - held * hq * L) < 1e-2 * held
    q = rotated(Q, b.origin[0, :held].tolist()).to(torch.bfloat16).double()
    kk = b.cache.read_kv(b.seqs[0])[0].double()
    total = torch.zeros(held, dtype=torch.float64, device="cuda")
    for layer in range(L):
        for h in range(hq):
            s = (q[layer, :, h] @ kk[layer, :, h // 2].t() * d ** -0.5).masked_fill(
                torch.arange(held, device="cuda")[None] > torch.arange(held, device="cuda")[:, None], -np.inf)
            total += torch.softmax(s, dim=1).sum(dim=0)
    assert (b.weights[0, :held].double() - total).abs().max().item() < 2e-3 * total.max().item()
    assert b.cache.device_status() == 0
