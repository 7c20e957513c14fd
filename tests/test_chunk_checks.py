"""Checks of the calls on chunks that need no device, of handles of a class derived from Handle."""
import pytest
import torch

from test_chunk_refusals import binding  # noqa: F401
from test_operator_refusals import Rows


def derived(b):
    class Named(b.Handle):
        pass

    h = Named(4096)
    h.layers, h.q_heads, h.kv_heads, h.head_dim, h.device = 2, 8, 2, 64, 0
    return h


def test_a_derived_handle_keeps_its_checks(binding):  # noqa: F811
    b, h = binding, derived(binding)
    q, k = Rows((5, 8, 64)), Rows((5, 2, 64))
    assert b._shape_of(h, k) == (8, 2, 64, 0) and b._width(h, "q_heads", None) == 512
    for bad in (lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], k, k, k, q, stream=0),              # rows of other heads
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], q, k, Rows((5, 2, 128)), q, stream=0),
                lambda: b.rlkv_paged_chunk_attention(h, 0, [0], [5], q, Rows((5, 2, 64), device=1), k, q, stream=0),
                lambda: b.rlkv_paged_append_chunks(h, 0, [0], [5], q, k, stream=0),
                lambda: b.rlkv_prompt_rotate(h, 0, q, q, None, q, k, stream=0)):
        with pytest.raises(ValueError):
            bad()


def test_the_stream_is_that_of_a_derived_handles_gpu(binding, monkeypatch):  # noqa: F811
    h = derived(binding)
    h.device = 3
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert binding._stream(None, h) == 103


def test_scratch_calls_refuse_without_a_handle(binding):  # noqa: F811
    for call in (lambda: binding.rlkv_paged_chunk_scratch_size(0), lambda: binding.rlkv_paged_set_chunk_scratch(0, None),
                 lambda: binding.rlkv_paged_set_chunk_scratch(0, 4096, 1 << 20)):
        with pytest.raises(binding.RlkvError) as e:
            call()
        assert e.value.code == binding.RLKV_EINVAL
