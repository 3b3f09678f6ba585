"""Attention with weights reads Q again after `out` is written: tensors that overlap are refused before anything runs."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import Both, bf16, refused

pytestmark = [pytest.mark.gpu, requires_cuda]

HQ, D, N = 4, 64, 40


@pytest.mark.parametrize("bits", [8, 16])
def test_overlapping_tensors_are_refused(bits):
    b = Both(1, 2, D, 16, bits=bits)
    s, t = b.new(), b.new()
    b.append([s, t], [90, 70])
    c = b.cache
    q0 = bf16(b.g.standard_normal((N, HQ, D)).astype(np.float32))[0]
    w = torch.zeros((2, 90), device="cuda")
    want = c.replay_attn_weights_batch([s, t], 0, q0, [0, 30, N], w)
    want_w, w = w, torch.zeros((2, 90), device="cuda")
    rows = torch.zeros((3 * N, HQ, D), device="cuda", dtype=torch.bfloat16)  # (memory that q, out and weights are cut from)
    q = rows[N: 2 * N]
    q.copy_(q0)
    call = lambda out, w: c.replay_attn_weights_batch([s, t], 0, q, [0, 30, N], w, out=out)  # noqa: E731
    launches = c.kernel_launches()
    for out in (q, rows[N - 1: 2 * N - 1], rows[1: N + 1], rows[2 * N - 1: 3 * N - 1]):
        refused("invalid", call, out, w)
    for at in (rows[0: N], rows[2 * N:]):                           # out beside q
        both = rows.view(-1).view(torch.float32)                    # 128 weights a row of q
        for first in (N * 128 - 1, N * 128, (2 * N - 1) * 128, at.storage_offset() // 2 - 1, at.storage_offset() // 2 + 500):
            first = min(max(first, 0), both.numel() - 180)
            refused("invalid", call, at, both[first: first + 180].view(2, 90))
    assert c.kernel_launches() == launches and torch.equal(q, q0) and bool((w == 0).all())
    for at in (rows[0: N], rows[2 * N:]):
        w.zero_()
        assert torch.equal(call(at, w), want) and torch.equal(w, want_w)
    # rows of weights on both sides of q and out, and a row that the call does not touch, over them
    big = torch.zeros((3, 3000 + 2 * N * HQ * D), device="cuda")
    inside = big[0, 100:].view(torch.bfloat16)[: 2 * N * HQ * D].view(2 * N, HQ, D)
    inside[:N].copy_(q0)
    weights = torch.as_strided(big, (2, 90), (big.stride(0), 1))
    c.replay_attn_weights_batch([s, t], 0, inside[:N], [0, 30, N], weights, out=inside[N:])
    assert torch.equal(weights, want_w) and torch.equal(inside[N:], want)
    refused("invalid", c.replay_attn_weights_batch, [s, t], 0, inside[:30], [0, 30, 30],
            torch.as_strided(big, (2, 90), (90, 1), 20), out=inside[N: N + 30])
    alone = c.replay_attn_weights_batch([s, t], 0, q0[:30], [0, 30, 30], torch.zeros((2, 90), device="cuda"))
    c.replay_attn_weights_batch([s, t], 0, inside[:30], [0, 30, 30], torch.as_strided(big, (2, 90), (95, 1), 0),
                                out=inside[N: N + 30])
    assert torch.equal(inside[N: N + 30], alone) and torch.equal(inside[:30], q0[:30])
    assert c.device_status() == 0
