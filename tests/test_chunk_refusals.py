"""Refusals of the calls on chunks and of the norms that need no device."""
import numpy as np
import pytest
import torch

from test_operator_refusals import Rows


@pytest.fixture(scope="module")
def binding():
    from paper_2510_08525_b200 import build
    build.build()
    import paper_2510_08525_b200.binding as b
    return b


def test_calls_refuse_without_a_handle(binding):
    b, lib = binding, binding.lib
    one = np.ones(1, np.int32).ctypes.data
    for call in (lambda: b.rlkv_paged_set_norms(0, 16, 16), lambda: b.rlkv_prompt_set_norms(0, 16, 16), lambda: b.rlkv_prompt_set_rotary(0, 16, 1, 128),
                 lambda: b.rlkv_paged_rotate_chunks(0, 0, [0], [1], 16, 16, 16, 16, stream=0),
                 lambda: b.rlkv_paged_chunk_attention(0, 0, [0], [1], 16, 16, 16, 16, stream=0),
                 lambda: b.rlkv_paged_append_chunks(0, 0, [0], [1], 16, 16, stream=0),
                 lambda: b.rlkv_paged_read(0, 0, [0], [0], [1], 16, 16, stream=0)):
        with pytest.raises(b.RlkvError) as e:
            call()
        assert e.value.code == b.RLKV_EINVAL
    assert lib.rlkv_prompt_rotate(0, 0, 16, 0, 16, 0, 1, 0, 16, 16, 0) == b.RLKV_EINVAL
    assert lib.rlkv_prompt_rotate_backward(0, 0, 16, 0, 16, 0, 1, 0, 16, 16, 16, 0, 16, 0, 0, 0, 0) == b.RLKV_EINVAL
    assert lib.rlkv_paged_chunk_attention(0, 0, one, 0, 1, 16, 0, 16, 0, 16, 0, 16, 0, 0) == b.RLKV_EINVAL


def handle(b):
    h = b.Handle(4096)
    h.layers, h.q_heads, h.kv_heads, h.head_dim, h.device = 2, 8, 2, 64, 0
    return h


def test_tensors_are_held_to_the_handle(binding):
    """Found before the library sees an address."""
    b, h = binding, handle(binding)
    q, k = Rows((5, 8, 64)), Rows((5, 2, 64))
    for bad in (lambda: b.rlkv_paged_chunk_attention(h, 0, [0, 1], [2], q, k, k, q, stream=0),           # no count for the second
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0, 1], [2, 4], q, k, k, q, stream=0),        # fewer tokens than counted
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], k, k, k, q, stream=0),              # rows of other heads
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], q, k, Rows((5, 2, 128)), q, stream=0),
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], q, Rows((5, 2, 64), device=1), k, q, stream=0),
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], Rows((5, 8, 64), size=4), k, k, q, stream=0),
                lambda: b.rlkv_paged_append_chunks(h, 0, [0], [5], q, k, stream=0),
                lambda: b.rlkv_paged_append_chunks(h, 0, [0], [5], k, Rows((5, 2, 64), stride=(0, 64, 1)), stream=0),
                lambda: b.rlkv_paged_rotate_chunks(h, 0, [0], [6], q, k, q, k, stream=0),
                lambda: b.rlkv_paged_read(h, 0, [0], [0, 1], [5], k, k, stream=0),
                lambda: b.rlkv_prompt_rotate(h, 0, q, k, torch.zeros(5, dtype=torch.int32), q, k, stream=0),   # positions on the host
                lambda: b.rlkv_prompt_rotate(h, 0, q, q, None, q, k, stream=0)):
        with pytest.raises(ValueError):
            bad()
    for w in (torch.ones(2, 64, dtype=torch.float64), torch.ones(1, 64)):
        with pytest.raises(ValueError):
            b.rlkv_paged_set_norms(h, w, None)
        with pytest.raises(ValueError):
            b.rlkv_prompt_set_norms(h, None, w)
