"""Strides of the norms' and rotation's rows, through the C entries: refused where they are out of range, taken up to the largest."""
import pytest
import torch

from test_gpu_norm_rotary import EPS, hz, rl, weights  # noqa: F401
from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu


def test_strides_out_of_range_are_refused(hz, rl, cuda_device):  # noqa: F811
    """Nothing is launched: the results stay as they are."""
    dev, n, Hq, Hkv, D = cuda_device, 3, 8, 2, 64
    p = hz.PromptAttention(1, Hkv, Hq, D, n, [1] * Hkv, 4, 60, device=dev)
    p.set_norms(*weights(1, D, 5, dev), EPS)
    q, k, y, z = (torch.full((n, h, D), 7.0, dtype=torch.bfloat16, device=dev) for h in (Hq, Hkv) * 2)
    dw = torch.full((2, D), 7.0, device=dev)
    bad = [(1 << 30) + 8, 1 << 40, 1 << 61, (1 << 63) - 8, -512, 8, 516]
    for s in bad:
        for qs, ks in ((s, 0), (0, s)):
            assert rl.lib.rlkv_prompt_rotate(p.handle, 0, q.data_ptr(), qs, k.data_ptr(), ks, n, 0, y.data_ptr(), z.data_ptr(), 0) == rl.RLKV_EINVAL
        for at in range(4):
            qs, ks, dqs, dks = (s if i == at else 0 for i in range(4))
            assert rl.lib.rlkv_prompt_rotate_backward(p.handle, 0, q.data_ptr(), qs, k.data_ptr(), ks, n, 0, y.data_ptr(), z.data_ptr(), y.data_ptr(), dqs,
                                                      z.data_ptr(), dks, dw[0].data_ptr(), dw[1].data_ptr(), 0) == rl.RLKV_EINVAL
    torch.cuda.synchronize()
    assert bool((y == 7).all()) and bool((z == 7).all()) and bool((dw == 7).all())


def test_a_far_stride(hz, rl, cuda_device):  # noqa: F811
    """Two tokens 2^30 elements apart (2 GB): the same bits as tokens behind one another."""
    dev, Hq, Hkv, D = cuda_device, 8, 2, 64
    p = hz.PromptAttention(1, Hkv, Hq, D, 2, [1] * Hkv, 4, 60, device=dev)
    p.set_norms(*weights(1, D, 5, dev), EPS)
    far = torch.zeros((1 << 30) + 4096, dtype=torch.bfloat16, device=dev)
    q, k = rand_bf16((2, Hq, D), 1).to(dev), rand_bf16((2, Hkv, D), 2).to(dev)
    wide_q, wide_k = (far[at:].as_strided((2, h, D), (1 << 30, D, 1)) for at, h in ((0, Hq), (1024, Hkv)))
    wide_q.copy_(q)
    wide_k.copy_(k)
    assert all(torch.equal(a, b) for a, b in zip(p.rotate(0, q, k), p.rotate(0, wide_q, wide_k)))
    dq_out, dk_out = rand_bf16((2, Hq, D), 3).to(dev), rand_bf16((2, Hkv, D), 4).to(dev)
    want = p.rotate_backward(0, q, k, dq_out, dk_out)
    dq, dk = (far[at:].as_strided((2, h, D), (1 << 30, D, 1)) for at, h in ((2048, Hq), (3328, Hkv)))
    dw = [torch.empty(D, device=dev) for _ in range(2)]
    rl.rlkv_prompt_rotate_backward(p.handle, 0, wide_q, wide_k, None, dq_out, dk_out, dq, dk, *dw)
    assert all(torch.equal(a, b) for a, b in zip(want, (dq, dk, *dw)))
