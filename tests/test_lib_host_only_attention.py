"""How attention calls on a host-only cache end: with the binding's or the library's refusal, as on any wrong argument."""
import pytest
import torch

import paper_2609_04875_gb300 as pe


@pytest.fixture(params=[8, 16])
def cache(request):
    c = pe.PagedKVCache(2, 2, 64, 16, 20, 4, 10, host_only=True, kv_bits=request.param)
    c.append_kv(c.seq_create(), n_tokens=20)
    return c


def test_attention_on_a_host_only_cache(cache):
    """The tensors a host-only cache could attend do not exist: the first one given is named."""
    q = torch.zeros((2, 4, 64), dtype=torch.bfloat16)
    for call in (lambda: cache.replay_attn(0, 0, q), lambda: cache.replay_attn_batch([0], 0, q, [0, 2]),
                 lambda: cache.replay_attn_static_scratch(0, 0, q)):
        with pytest.raises(TypeError, match="Q must be a CUDA tensor"):
            call()
    with pytest.raises(ValueError, match="host-only"):
        cache.replay_attn_weights_batch([0], 0, q, [0, 2], torch.zeros((1, 20)))
    with pytest.raises(ValueError, match="host-only"):
        cache.read_kv_batch([0], [0], [0, 2])
