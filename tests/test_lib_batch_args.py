"""What the binding refuses before the library reads the host arrays of a batch call: offsets fewer than the sequences
need."""
import numpy as np
import pytest
import torch

import paper_2609_04875_gb300 as pe


@pytest.fixture(params=[8, 16])
def cache(request):
    c = pe.PagedKVCache(2, 2, 64, 16, 20, 4, 10, host_only=True, kv_bits=request.param)
    for _ in range(3):
        c.append_kv(c.seq_create(), n_tokens=20)
    return c


def tensors(rows, dtype=torch.bfloat16):
    return torch.zeros((rows, 4, 64), dtype=dtype)


@pytest.mark.parametrize("cu", [[0], [0, 1], [0, 1, 2], [0, 1, 2, 9, 4]])
def test_short_offsets(cache, cu):
    """Too few, or more than enough but with the last one read past the tensors' rows."""
    seqs, n = [0, 1, 2], cu[-1]
    q, w = tensors(n), torch.zeros((3, 20))
    kv = torch.zeros((2, n, 2, 64), dtype=torch.bfloat16)
    before = cache.free_list(), [cache.seq_info(s) for s in seqs]
    for call in (lambda: cache.replay_attn_batch(seqs, 0, q, cu, out=q.clone()),
                 lambda: cache.replay_attn_batch(seqs, 0, q, cu),
                 lambda: cache.prepare_replay_attn_batch(seqs, 0, q, cu, q.clone()),
                 lambda: cache.replay_attn_weights_batch(seqs, 0, q, cu, w, out=q.clone()),
                 lambda: cache.replay_attn_weights_batch(seqs, 0, q, cu, w),
                 lambda: cache.append_kv_batch(seqs, cu_tokens=cu),
                 lambda: cache.append_kv_batch(seqs, kv, kv, cu),
                 lambda: cache.prepare_append_kv_batch(seqs, kv, kv, cu),
                 lambda: cache.replay_rounds(seqs, np.zeros((1, 3), dtype=np.int32), cu),
                 lambda: cache.read_kv_batch(seqs, [0, 0, 0], cu)):
        with pytest.raises(ValueError, match="cu"):
            call()
    assert (cache.free_list(), [cache.seq_info(s) for s in seqs]) == before


def test_weights_take_one_offset_more_than_sequences(cache):
    with pytest.raises(ValueError, match="cu_q"):
        cache.replay_attn_weights_batch([0], 0, tensors(2), [0, 1, 2], torch.zeros((1, 20)))


def test_short_crops(cache):
    for call in (cache.crop_batch, cache.prepare_crop_batch):
        with pytest.raises(ValueError, match="taus"):
            call([0, 1, 2], [5, 5])
    assert [cache.seq_info(s)[0] for s in range(3)] == [20, 20, 20]


def test_as_many_as_needed_go_through(cache):
    cache.append_kv_batch([0, 1], cu_tokens=[0, 1, 3])
    cache.append_kv_batch([0], cu_tokens=[0, 2, 9])            # (what stands past the last sequence's is not read)
    cache.append_kv_batch([], cu_tokens=[])
    cache.replay_rounds([0, 1], np.ones((1, 2), dtype=np.int32), [0, 1, 2])
    cache.crop_batch([0, 1], [3, 4])
    cache.prepare_crop_batch([0, 1], [3, 4])()
    assert [cache.seq_info(s)[0] for s in range(3)] == [2, 3, 20]
