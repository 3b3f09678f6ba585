"""Outputs that a call makes itself for another stream than the current one: memory that the current stream may still be
using is not written, and an output's memory is not given out again before the current stream is done with it."""
import numpy as np
import pytest
import torch

from gpu_common import requires_cuda
from test_gpu_q8 import Both, bf16

pytestmark = [pytest.mark.gpu, requires_cuda]

L, HQ, HKV, D, T = 2, 8, 2, 64, 600


def calls(b, s, q, w):
    """(name, call with stream=, the tensors it makes)"""
    c = b.cache
    qs = q[:4].expand(L, 4, HQ, D).contiguous()
    k = torch.zeros((L, 4, HKV, D), device="cuda", dtype=torch.bfloat16)
    return [
        ("replay_attn", lambda st: [c.replay_attn(s, 1, q, stream=st)]),
        ("replay_attn_batch", lambda st: [c.replay_attn_batch([s], 1, q, [0, q.shape[0]], stream=st)]),
        ("replay_attn_weights_batch", lambda st: [c.replay_attn_weights_batch([s], 1, q, [0, q.shape[0]], w, stream=st)]),
        ("static scratch", lambda st: [c.replay_attn_static_scratch(s, 1, q, stream=st)]),
        ("read_kv", lambda st: list(c.read_kv(s, 0, T, stream=st))),
        ("rounds", lambda st: [c.replay_rounds([s], np.array([[4]], dtype=np.int32), [0, 4], k, k, qs, stream=st)]),
        ("evict_batch", lambda st: [c.evict_batch([s], [c.seq_info(s)[0] - 1], w, stream=st)]),
    ]


@pytest.mark.parametrize("which", ["stream", "handle"])
def test_outputs_of_another_stream(which):
    b = Both(L, HKV, D, 16, pages=120)
    s = b.new()
    b.append([s], [T])
    q = bf16(b.g.standard_normal((100, HQ, D)).astype(np.float32))[0]
    w = torch.zeros((1, 700), device="cuda")
    side = torch.cuda.Stream()
    given = side if which == "stream" else side.cuda_stream
    for name, call in calls(b, s, q, w):
        torch.cuda.synchronize()
        out = call(given)
        torch.cuda.synchronize()
        sizes = [t.numel() * t.element_size() for t in out]
        mine = [t.data_ptr() for t in out]
        torch.cuda._sleep(20_000_000)               # work of the current stream, some ms, that stands for a use of them
        del out
        with torch.cuda.stream(side):
            others = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes]
        if not torch.cuda.current_stream().query():
            assert not set(mine) & {t.data_ptr() for t in others}, name
        torch.cuda.synchronize()
        # blocks that the current stream has freed, of the outputs' sizes
        freed = [torch.empty(n, dtype=torch.uint8, device="cuda") for n in sizes * 3]
        ptrs = {t.data_ptr() for t in freed}
        del freed, others
        assert not ptrs & {t.data_ptr() for t in call(given)}, name
        torch.cuda.synchronize()
    assert b.cache.device_status() == 0


def test_what_they_hold():
    """The same values as on the current stream, and on the default stream named by its handle."""
    b = Both(L, HKV, D, 16, pages=120)
    s = b.new()
    b.append([s], [T])
    q = bf16(b.g.standard_normal((100, HQ, D)).astype(np.float32))[0]
    w = torch.zeros((1, 700), device="cuda")
    side = torch.cuda.Stream()
    for name, call in calls(b, s, q, w)[:5]:
        want = call(None)
        torch.cuda.synchronize()
        for given in (side, side.cuda_stream, torch.cuda.default_stream(), 0):
            got = call(given)
            torch.cuda.synchronize()
            assert all(torch.equal(x, y) for x, y in zip(got, want)), name
