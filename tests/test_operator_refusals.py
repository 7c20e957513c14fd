"""Refusals of the rotation, score and prompt calls that need no device."""
import numpy as np
import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2510_08525_b200 import build
    build.build()
    import paper_2510_08525_b200.binding as b
    return b


def test_rotation_and_score_calls_refuse_without_a_device(binding):
    b, lib = binding, binding.lib
    f = np.ones(64)
    for call in (lambda: b.rlkv_paged_set_rotary(0, 16, 10, 128), lambda: b.rlkv_paged_set_scores(0, 1.0),
                 lambda: b.rlkv_paged_append_rotated(0, 0, [0], 16, 16, 16, 16, stream=0),
                 lambda: b.rlkv_paged_prefill_rotated(0, 0, 0, 16, 16, 16, 1, 16, stream=0),
                 lambda: b.rlkv_rotary_table(f, 0, 16, stream=0), lambda: b.rlkv_rotary_table(f, 10, 8, stream=0),
                 lambda: b.rlkv_rotary_table(np.ones(65), 10, 16, stream=0), lambda: b.rlkv_rotary_table(f, 10, None, stream=0)):
        with pytest.raises(b.RlkvError) as e:
            call()
        assert e.value.code == b.RLKV_EINVAL
    assert lib.rlkv_rotary_table(f.ctypes.data, 3, 10, 16, 0) == b.RLKV_EINVAL


def test_prompt_calls_refuse_without_a_device(binding):
    b, lib = binding, binding.lib
    m = np.ones(2, np.uint8)
    for call in (lambda: b.rlkv_prompt_destroy(0), lambda: b.rlkv_prompt_kernel_status(0),
                 lambda: b.rlkv_prompt_create(1, 2, 8, 96, 10, m, 4, 60), lambda: b.rlkv_prompt_create(1, 2, 8, 128, 0, m, 4, 60),
                 lambda: b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 0), lambda: b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 60, -1.0)):
        with pytest.raises(b.RlkvError) as e:
            call()
        assert e.value.code == b.RLKV_EINVAL
    with pytest.raises(ValueError):
        b.rlkv_prompt_create(1, 2, 8, 128, 10, [1], 4, 60)
    with pytest.raises(ValueError):
        b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 60, 0.0, np.ones(7))
    assert lib.rlkv_prompt_attention(0, 0, 16, 0, 16, 0, 16, 0, 1, 1, 16, 0, 1, 0, 16, 16, 0) == b.RLKV_EINVAL
    assert lib.rlkv_prompt_attention_backward(0, 0, 16, 0, 16, 0, 16, 0, 1, 1, 16, 0, 1, 0, 16, 16, 16, 16, 16, 16, 0) == b.RLKV_EINVAL
