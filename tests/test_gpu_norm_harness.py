"""PromptAttention.rotate and rotate_backward as a model calls them: whichever of rotation and norms it has, with and without positions."""
import pytest
import torch

from test_gpu_norm_rotary import EPS, backward64, check_forward, hz, weights  # noqa: F401
from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("norms,rot", [("qk", 128), ("q", 128), ("k", 64), ("", 128), ("q", 0), ("k", 0)])
def test_gradients_of_the_norms_that_are_set(hz, cuda_device, norms, rot):  # noqa: F811
    """The default call returns the gradient of each norm that is set and None of the others (tolerances: test_gpu_norm_rotary)."""
    dev, n, Hq, Hkv, D = cuda_device, 70, 8, 2, 128
    p = hz.PromptAttention(1, Hkv, Hq, D, n, [1] * Hkv, 4, 60, device=dev)
    if rot:
        p.set_rotary(hz.rotary_table(n, rot, device=dev), rot)
    qw, kw = weights(1, D, 5, dev)
    qw, kw = qw if "q" in norms else None, kw if "k" in norms else None
    p.set_norms(qw, kw, EPS)
    q, k = rand_bf16((n, Hq, D), 1).to(dev), rand_bf16((n, Hkv, D), 2).to(dev)
    dq_out, dk_out = rand_bf16((n, Hq, D), 3).to(dev), rand_bf16((n, Hkv, D), 4).to(dev)
    dq, dk, dqw, dkw = p.rotate_backward(0, q, k, dq_out, dk_out)
    pos = torch.arange(n).numpy()
    for x, w, dy, dx, dw in ((q, qw, dq_out, dq, dqw), (k, kw, dk_out, dk, dkw)):
        want, size, want_w, size_w = backward64(x, None if w is None else w[0], pos, rot, False, dy)
        assert bool(((dx.double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size + 2.0 ** -133).all())
        assert (dw is None) == (w is None)
        if w is not None:
            terms = x.shape[0] * x.shape[1]
            assert bool(((dw.double().cpu() - want_w).abs() <= ((terms / 256 + 32) * 2.0 ** -24 + 2.0 ** -19) * size_w + 1e-30).all())
    assert all(torch.equal(a, b) for a, b in zip(p.rotate_backward(0, q, k, dq_out, dk_out, weights=False), (dq, dk)))


@pytest.mark.parametrize("rows,given", [(100, False), (100, True), (33, False), (33, True), (0, False), (0, True)])
def test_rows_of_no_document_are_zero(hz, cuda_device, rows, given):  # noqa: F811
    """Tokens past the table's rows (0: no rotation, no limit) or at negative positions, forward and backward, in memory that held NaN."""
    dev, n, Hq, Hkv, D = cuda_device, 70, 8, 2, 128
    p = hz.PromptAttention(1, Hkv, Hq, D, n, [1] * Hkv, 4, 60, device=dev)
    if rows:
        p.set_rotary(hz.rotary_table(rows, D, device=dev), D)
    w = weights(1, D, 5, dev)
    p.set_norms(*w, EPS)
    pos = torch.arange(n)
    if given:
        pos[3], pos[50] = -1, -5
    mine = (pos >= 0) & (pos < (rows or n))
    q, k = rand_bf16((n, Hq, D), 1).to(dev), rand_bf16((n, Hkv, D), 2).to(dev)
    dy = rand_bf16((n, Hq, D), 3).to(dev), rand_bf16((n, Hkv, D), 4).to(dev)
    dirt = [torch.full((n, h, D), float("nan"), dtype=torch.bfloat16, device=dev) for h in (Hq, Hkv) * 4]
    del dirt
    at = pos.to(dev, torch.int32) if given else None
    out = p.rotate(0, q, k, at)
    grads = p.rotate_backward(0, q, k, *dy, at)
    for x, y, dx, g, wt in zip((q, k), out, grads, dy, w):
        check_forward(y[mine], x[mine], wt[0], pos[mine].numpy(), D if rows else 0, False)
        want, size, _, _ = backward64(x[mine], wt[0], pos[mine].numpy(), D if rows else 0, False, g[mine])
        assert bool(((dx[mine].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -19 * size + 2.0 ** -133).all())
        assert bool((y[~mine] == 0).all()) and bool((dx[~mine] == 0).all())


def test_nothing_is_cleared_that_the_kernels_write(hz, cuda_device, monkeypatch):  # noqa: F811
    """Every token at its own index and inside the table: the results are not cleared in front of the launches."""
    dev, n = cuda_device, 64
    p = hz.PromptAttention(1, 2, 8, 128, n, [1, 0], 4, 60, device=dev)
    q, k = rand_bf16((n, 8, 128), 1).to(dev), rand_bf16((n, 2, 128), 2).to(dev)
    w = weights(1, 128, 5, dev)
    table = hz.rotary_table(n, 128, device=dev)
    monkeypatch.setattr(torch, "zeros", None)
    p.set_norms(*w, EPS)
    p.rotate_backward(0, q, k, *p.rotate(0, q, k))
    p.set_rotary(table, 128)
    p.rotate_backward(0, q, k, *p.rotate(0, q, k))
