"""Norms of query and key heads with their rotation: on packed tokens with gradients (rlkv_prompt_rotate,
rlkv_prompt_rotate_backward), and in the rotated calls of the paged cache (rlkv_paged_set_norms), against the formulas in 64 bits.

Tolerances.  u = x / sqrt(mean x^2 + eps) in fp32: a sum of D squares, (D + 2) 2^-24 at the very worst and half of it in the
root, the root's 2^-22 and three products -- 2^-18 for 128 elements in the worst order, and the sums here are trees of depth 20 -- 2^-20
of the magnitudes |a| + |b| that a rotation adds; bf16 once, 2^-8 of the value.  Gradients: dx = r (g - u mean(g u)) with the same
relative errors of g, u and the mean: 2^-19 r (|g| + |u| mean|g u|), then 2^-8 of the value.  dw is a sum of n terms in fp32, n / 256
of them one after the other at the worst: (n / 256 + 32) 2^-24 of the sum of their magnitudes, and 2^-19 of it for the terms' own errors."""
import numpy as np
import pytest
import torch

from test_gpu_parity import rand_bf16
from test_gpu_rotary import check_bf16, inv_freq, rotate64, same_state

pytestmark = pytest.mark.gpu
EPS = 1e-6


@pytest.fixture(scope="module")
def rl(cuda_device):
    import paper_2510_08525_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def hz(cuda_device):
    import paper_2510_08525_b200.harness as harness
    return harness


def weights(layers, D, seed, dev):
    g = torch.Generator().manual_seed(seed)
    return [(1 + 0.3 * torch.randn((layers, D), generator=g)).to(dev) for _ in range(2)]


def normed(x, w, eps=EPS):
    return x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps) * w


def forward64(x, w, pos, rot, interleaved, eps=EPS):
    """y and |a| + |b| of every element's pair."""
    x = x.double().cpu()
    y = x if w is None else normed(x, w.double().cpu(), eps)
    return rotate64(y, pos, rot, interleaved) if rot else (y, torch.zeros_like(y))


def check_forward(got, x, w, pos, rot, interleaved, eps=EPS):
    want, size = forward64(x, w, pos, rot, interleaved, eps)
    err = (got.double().cpu() - want).abs()
    bound = 2.0 ** -8 * want.abs() + 2.0 ** -20 * (size + want.abs()) + 2.0 ** -133
    assert bool((err <= bound).all()), float((err / bound).max())


def backward64(x, w, pos, rot, interleaved, dy, eps=EPS):
    """dx, its bound's size, dw and the sum of its terms' magnitudes, from the formula."""
    x, dy = x.double().cpu(), dy.double().cpu()
    h, size = rotate64(dy, -np.asarray(pos, np.float64), rot, interleaved) if rot else (dy, torch.zeros_like(dy))
    if w is None:
        return h, size + h.abs(), None, None
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    u, g = x * r, h * w.double().cpu()
    dx = r * (g - u * (g * u).mean(-1, keepdim=True))
    bound = r * (g.abs() + size * w.double().cpu().abs() + u.abs() * (g * u).abs().mean(-1, keepdim=True))
    return dx, bound, (h * u).sum((0, 1)), (h * u).abs().sum((0, 1))


CASES = [
    # Hkv, Hq, D, tokens, rot, interleaved, norms of q and k, slices, with positions
    (8, 32, 128, 1, 128, False, "qk", True, True), (2, 8, 64, 3, 64, True, "qk", False, True), (4, 28, 128, 33, 64, False, "qk", True, False),
    (1, 1, 128, 257, 128, False, "q", False, True), (3, 24, 64, 500, 32, False, "k", True, True), (2, 2, 128, 40, 0, False, "qk", False, True),
    (2, 16, 128, 100, 128, True, "", True, True), (8, 32, 128, 3000, 128, False, "qk", True, True), (128, 1024, 64, 5, 64, False, "qk", False, True),
    (1, 3, 64, 1, 0, False, "q", False, False), (5, 5, 128, 70, 16, True, "qk", True, True)]


@pytest.mark.parametrize("Hkv,Hq,D,n,rot,interleaved,norms,sliced,positions", CASES)
def test_prompt_rotate_and_gradients(hz, rl, cuda_device, Hkv, Hq, D, n, rot, interleaved, norms, sliced, positions):
    dev, rows = cuda_device, 4096
    p = hz.PromptAttention(2, Hkv, Hq, D, n, [1] * 2 * Hkv, 4, 60, device=dev)
    if rot:
        p.set_rotary(hz.rotary_table(rows, rot, device=dev), rot, interleaved)
    qw, kw = weights(2, D, 3, dev)
    qw, kw = qw if "q" in norms else None, kw if "k" in norms else None
    p.set_norms(qw, kw, EPS)
    x = rand_bf16((n, Hq + 2 * Hkv, D), 11).to(dev)
    x[n // 2] *= 100.0
    x[n // 3, 0] = 0.0     # a row of zeros
    q, k = x[:, :Hq], x[:, Hq:Hq + Hkv]
    if not sliced:
        q, k = q.contiguous(), k.contiguous()
    pos = np.arange(n)
    at = None
    if positions:          # documents behind one another, some tokens of none
        pos = (np.arange(n) * 7 + 3) % (rows if rot else 10 ** 6)
        pos[n // 4] = -1 if n > 3 else pos[n // 4]
        if rot and n > 10:
            pos[n // 5] = rows
        at = torch.from_numpy(pos.astype(np.int32)).to(dev)
    mine = torch.from_numpy((pos >= 0) & (pos < rows if rot else True))
    q_out, k_out = (torch.full((n + 1, h, D), 7.0, dtype=torch.bfloat16, device=dev) for h in (Hq, Hkv))
    rl.rlkv_prompt_rotate(p.handle, 1, q, k, at, q_out, k_out)
    dq_out, dk_out = rand_bf16((n, Hq, D), 21).to(dev), rand_bf16((n, Hkv, D), 22).to(dev)
    wide = torch.full((n + 1, Hq + 2 * Hkv, D), 7.0, dtype=torch.bfloat16, device=dev)   # the gradient of the projection's output
    dw = [None if w is None else torch.full((D + 1,), 7.0, device=dev) for w in (qw, kw)]
    rl.rlkv_prompt_rotate_backward(p.handle, 1, q, k, at, dq_out, dk_out, wide[:n, :Hq], wide[:n, Hq:Hq + Hkv], *dw)
    for got, x, w, dy, dx, d in ((q_out, q, qw, dq_out, wide[:, :Hq], dw[0]), (k_out, k, kw, dk_out, wide[:, Hq:Hq + Hkv], dw[1])):
        w = None if w is None else w[1]
        check_forward(got[:n][mine], x[mine], w, pos[mine.numpy()], rot, interleaved)
        assert bool((got[:n][~mine] == 7).all()) and bool((got[n] == 7).all())
        want, size, want_w, size_w = backward64(x[mine], w, pos[mine.numpy()], rot, interleaved, dy[mine])
        err = (dx[:n][mine].double().cpu() - want).abs()
        bound = 2.0 ** -8 * want.abs() + 2.0 ** -19 * size + 2.0 ** -133
        assert bool((err <= bound).all()), float((err / bound).max())
        assert bool((dx[:n][~mine] == 7).all()) and bool((dx[n] == 7).all())
        if d is not None:
            err = (d[:D].double().cpu() - want_w).abs()
            terms = x[mine].shape[0] * x.shape[1]
            assert bool((err <= ((terms / 256 + 32) * 2.0 ** -24 + 2.0 ** -19) * size_w + 1e-30).all()), float((err / size_w).max())
            assert float(d[D]) == 7
    assert bool((wide[:, Hq + Hkv:] == 7).all())
    # the same bits again, and without the weights' gradients
    again = torch.full_like(wide, 7.0)
    rl.rlkv_prompt_rotate_backward(p.handle, 1, q, k, at, dq_out, dk_out, again[:n, :Hq], again[:n, Hq:Hq + Hkv])
    assert torch.equal(wide, again)
    dw2 = [None if w is None else torch.empty_like(w) for w in dw]
    rl.rlkv_prompt_rotate_backward(p.handle, 1, q, k, at, dq_out, dk_out, again[:n, :Hq], again[:n, Hq:Hq + Hkv], *dw2)
    assert all(a is None or torch.equal(a[:D], b[:D]) for a, b in zip(dw, dw2))


@pytest.mark.parametrize("D,rot,interleaved", [(64, 64, False), (128, 64, True)])
def test_gradients_against_differences(hz, cuda_device, D, rot, interleaved):
    """Along random directions: the derivative of sum(y * dy) by central differences in 64 bits (h = 1e-4: off by h^2 = 1e-8 times a
    third derivative of order one) against the kernel's gradients, whose rounding to bf16 is at most 2^-8 of each product."""
    dev, n, Hq, Hkv = cuda_device, 17, 4, 2
    p = hz.PromptAttention(1, Hkv, Hq, D, n, [1] * Hkv, 4, 60, device=dev)
    p.set_rotary(hz.rotary_table(64, rot, device=dev), rot, interleaved)
    qw, kw = weights(1, D, 5, dev)
    p.set_norms(qw, kw, EPS)
    q, k = rand_bf16((n, Hq, D), 1).to(dev), rand_bf16((n, Hkv, D), 2).to(dev)
    dq_out, dk_out = rand_bf16((n, Hq, D), 3).to(dev), rand_bf16((n, Hkv, D), 4).to(dev)
    dq, dk, dqw, dkw = p.rotate_backward(0, q, k, dq_out, dk_out)
    pos, h = np.arange(n), 1e-4
    for x, w, dy, dx, dw in ((q, qw, dq_out, dq, dqw), (k, kw, dk_out, dk, dkw)):
        x, w, dy, dx, dw = (y.double().cpu() for y in (x, w[0], dy, dx, dw))
        value = lambda x, w: float((rotate64(normed(x, w), pos, rot, interleaved)[0] * dy).sum())  # noqa: E731
        g = torch.Generator().manual_seed(6)
        for _ in range(4):
            a, b = torch.randn(x.shape, generator=g, dtype=torch.float64), torch.randn(w.shape, generator=g, dtype=torch.float64)
            slope = (value(x + h * a, w) - value(x - h * a, w)) / (2 * h)
            assert abs(slope - float((dx * a).sum())) <= 2.0 ** -8 * float((dx * a).abs().sum()) + 1e-4
            slope = (value(x, w + h * b) - value(x, w - h * b)) / (2 * h)
            assert abs(slope - float((dw * b).sum())) <= 2.0 ** -18 * float((dw * b).abs().sum()) + 1e-3


def test_in_place_and_captured(hz, rl, cuda_device):
    dev, n = cuda_device, 130
    p = hz.PromptAttention(1, 2, 8, 128, n, [1, 0], 4, 60, device=dev)
    p.set_rotary(hz.rotary_table(200, 128, device=dev), 128)
    p.set_norms(*weights(1, 128, 5, dev), EPS)
    q, k = rand_bf16((n, 8, 128), 1).to(dev), rand_bf16((n, 2, 128), 2).to(dev)
    want = p.rotate(0, q, k)
    a, b = q.clone(), k.clone()
    rl.rlkv_prompt_rotate(p.handle, 0, a, b, None, a, b)
    assert torch.equal(a, want[0]) and torch.equal(b, want[1])
    grads = p.rotate_backward(0, q, k, *want)
    a, b = want[0].clone(), want[1].clone()
    rl.rlkv_prompt_rotate_backward(p.handle, 0, q, k, None, a, b, a, b)
    assert torch.equal(a, grads[0]) and torch.equal(b, grads[1])
    # forward and backward in one graph, replayed on other inputs and positions
    pos = torch.arange(n, dtype=torch.int32, device=dev)
    outs = [torch.empty_like(x) for x in (q, k, q, k)] + [torch.empty(128, device=dev) for _ in range(2)]
    run = lambda: (rl.rlkv_prompt_rotate(p.handle, 0, q, k, pos, outs[0], outs[1]),  # noqa: E731
                   rl.rlkv_prompt_rotate_backward(p.handle, 0, q, k, pos, outs[0], outs[1], *outs[2:]))
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(3):
        q.copy_(rand_bf16((n, 8, 128), 50 + seed))
        k.copy_(rand_bf16((n, 2, 128), 60 + seed))
        pos.copy_(torch.randint(0, 200, (n,), generator=torch.Generator().manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in outs]
        for x in outs:
            x.zero_()
        run()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for x, y in zip(got, outs))


@pytest.mark.parametrize("Hkv,Hq,D,mask,S,W,rot,interleaved,fp8,norms", [
    (2, 8, 64, "10", 4, 60, 64, False, False, "qk"), (4, 28, 128, "1001", 16, 112, 128, False, False, "qk"),
    (4, 28, 128, "0110", 16, 112, 64, False, True, "qk"), (3, 24, 128, "010", 4, 60, 128, True, True, "k"), (1, 1, 128, "0", 0, 5, 128, True, False, "q")])
def test_normed_prefill_and_append(hz, rl, cuda_device, Hkv, Hq, D, mask, S, W, rot, interleaved, fp8, norms):
    """The rotated calls with norms set: q_out and k_out against the formula; a prompt's cache bytes against the plain append of k_out
    (16 bits), and every row read back against the formula, rounded to bf16, or to a code."""
    dev, lens = cuda_device, [70, 1, 300]
    scale = ([0.01 + 0.003 * h for h in range(Hkv)], [0.02 + 0.001 * h for h in range(Hkv)]) if fp8 else (None, None)
    cache, plain = (hz.PagedCache(1, Hkv, Hq, D, 3, 12, 400, [int(c) for c in mask], S, W, device=dev, k_scale=scale[0], v_scale=scale[1])
                    for _ in range(2))
    cache.set_rotary(hz.rotary_table(400, rot, device=dev), rot, interleaved)
    qw, kw = weights(1, D, 9, dev)
    qw, kw = qw if "q" in norms else None, kw if "k" in norms else None
    cache.set_norms(qw, kw, EPS)
    w = [None if x is None else x[0] for x in (qw, kw)]
    a, b = [cache.open_seq() for _ in lens], [plain.open_seq() for _ in lens]
    exact, size = [], []
    for s, t, n in zip(a, b, lens):
        x = rand_bf16((n, Hq + 2 * Hkv, D), n).to(dev)
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        q_out, k_out = cache.prefill_rotated(0, s, q, k, v)
        check_forward(q_out, q, w[0], np.arange(n), rot, interleaved)
        check_forward(k_out, k, w[1], np.arange(n), rot, interleaved)
        want = forward64(k, w[1], np.arange(n), rot, interleaved)
        exact.append(want[0])
        size.append(want[1])
        plain.prefill(0, t, k_out, v.contiguous())
    if not fp8:
        for s, t in zip(a, b):
            same_state(cache, plain, s, t)
    for step in range(3):
        x = rand_bf16((3, Hq + 2 * Hkv, D), 1000 + step).to(dev)
        q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
        pos = np.array(lens) + step
        other_q, other_k = cache.rotate_chunks(0, a, [1, 1, 1], q, k)     # the same rotation, before it is appended
        check_forward(other_q, q, w[0], pos, rot, interleaved)
        check_forward(other_k, k, w[1], pos, rot, interleaved)
        check_forward(cache.append_rotated(0, a, q, k, v), q, w[0], pos, rot, interleaved)
        want = forward64(k, w[1], pos, rot, interleaved)
        exact, size = ([torch.cat([old, y[i:i + 1]]) for i, old in enumerate(kept)] for kept, y in ((exact, want[0]), (size, want[1])))
    k, _ = cache.read(0, a, [0, 0, 0], [n + 3 for n in lens])
    for got, want, pairs, n in zip(k.cpu().split([n + 3 for n in lens]), exact, size, lens):
        t = torch.arange(n + 3)
        for h in range(Hkv):
            held = (t < S) | (t >= n + 3 - W) if mask[h] == "0" else t >= 0
            x = want[held, h]
            if fp8:
                s = scale[0][h]
                x = x.clamp(-448 * s, 448 * s)  # (codes saturate there)
                # half a step of E4M3 (2^-4 of the value, 2^-10 below its normal range), what fp32 is off by, and bf16 when read back
                bound = (2.0 ** -4 + 2.0 ** -7) * x.abs() + 2.0 ** -10 * s
            else:
                bound = 2.0 ** -8 * x.abs() + 2.0 ** -20 * (pairs[held, h] + x.abs()) + 2.0 ** -133
            assert bool(((got[held, h].double() - x).abs() <= bound).all())


def test_norms_with_attention_and_its_gradients(hz, cuda_device):
    """Training: norms and rotation, attention over packed documents, and all the way back to the projections and the weights, against
    autograd in 64 bits.  Between the two, rows are rounded to bf16 (q, k, out, dq, dk: 2^-8 of each): the gradients' norms are within
    four such roundings, 2^-6, of their own norms."""
    dev, Hkv, Hq, D, S, W = cuda_device, 2, 8, 64, 4, 60
    lens = [70, 1, 200]
    n = sum(lens)
    p = hz.PromptAttention(1, Hkv, Hq, D, n, [1, 0], S, W, device=dev)
    p.set_rotary(hz.rotary_table(256, D, device=dev), D)
    qw, kw = weights(1, D, 5, dev)
    p.set_norms(qw, kw, EPS)
    x = rand_bf16((n, Hq + 2 * Hkv, D), 1).to(dev)
    q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    pos = torch.cat([torch.arange(m) for m in lens])
    at, starts = pos.to(dev, torch.int32), torch.tensor([0, 70, 71, 271], dtype=torch.int32, device=dev)
    dout = rand_bf16((n, Hq, D), 2).to(dev)
    qr, kr = p.rotate(0, q, k, at)
    out, lse = p.forward(0, qr, kr, v, starts)
    dqr, dkr, dv = p.backward(0, qr, kr, v, out, lse, dout, starts)
    dq, dk, dqw, dkw = p.rotate_backward(0, q, k, dqr, dkr, at)
    leaves = [y.double().cpu().clone().requires_grad_() for y in (q, k, v, qw[0], kw[0])]
    a, b, c, wa, wb = leaves
    ang = pos.double()[:, None, None] * torch.from_numpy(inv_freq(D))

    def turned(y):
        e, f = y[..., :D // 2], y[..., D // 2:]
        return torch.cat([e * ang.cos() - f * ang.sin(), f * ang.cos() + e * ang.sin()], -1)

    a, b = turned(normed(a, wa)), turned(normed(b, wb))
    s = torch.einsum("ihgd,jhd->hgij", a.view(n, Hkv, Hq // Hkv, D), b) / D ** 0.5
    doc = torch.repeat_interleave(torch.arange(3), torch.tensor(lens))
    seen = (doc[:, None] == doc) & (pos[:, None] >= pos)
    seen = torch.stack([seen, seen & ((pos < S) | (pos[:, None] - pos < W))])[:, None]
    o = torch.einsum("hgij,jhd->ihgd", torch.softmax(s.masked_fill(~seen, -1e300), -1), c).reshape(n, Hq, D)
    want = torch.autograd.grad(o, leaves, dout.double().cpu())
    for got, ref in zip((dq, dk, dv, dqw, dkw), want):
        assert float((got.double().cpu() - ref).norm()) <= 2.0 ** -6 * float(ref.norm())


def test_refusals(hz, rl, cuda_device):
    dev = cuda_device
    p = hz.PromptAttention(2, 2, 8, 64, 10, [1] * 4, 4, 60, device=dev)
    q, k = rand_bf16((10, 8, 64), 1).to(dev), rand_bf16((10, 2, 64), 2).to(dev)
    with pytest.raises(rl.RlkvError) as e:      # neither rotation nor norms
        p.rotate(0, q, k)
    assert e.value.code == rl.RLKV_EINVAL
    w = torch.ones((2, 64), device=dev)
    for bad in (lambda: p.set_norms(w[0], w), lambda: p.set_norms(w.half(), w), lambda: p.set_norms(w, w, 0.0), lambda: p.set_norms(w, w, 1.5),
                lambda: rl.rlkv_prompt_set_norms(p.handle, w.data_ptr() + 4, w), lambda: rl.rlkv_prompt_set_norms(p.handle, w.cpu(), w),
                lambda: p.set_rotary(hz.rotary_table(8, 128, device=dev), 128), lambda: rl.rlkv_prompt_set_rotary(p.handle, w, 1, 72)):
        with pytest.raises((ValueError, rl.RlkvError)):
            bad()
    p.set_norms(w, None)
    out = p.rotate(1, q, k)
    assert torch.equal(out[1], k)               # no norm and no rotation of the keys
    ok = dict(layer=0, q=q, k=k, at=None, dq_out=q, dk_out=k, dq=torch.empty_like(q), dk=torch.empty_like(k), dqw=torch.empty(64, device=dev), dkw=None)
    call = lambda **x: rl.rlkv_prompt_rotate_backward(p.handle, *{**ok, **x}.values())  # noqa: E731
    call()
    short = torch.zeros(9, dtype=torch.int32, device=dev)
    for bad in (dict(layer=2), dict(dkw=torch.empty(64, device=dev)), dict(dq=None), dict(at=short), dict(at=torch.zeros(10, device=dev)),
                dict(dqw=torch.empty(63, device=dev)), dict(dqw=torch.empty(64, dtype=torch.float64, device=dev)), dict(dq_out=q[:9]),
                dict(q=rand_bf16((11, 8, 64), 1).to(dev)), dict(k=q), dict(dk=k[:9]), dict(q=q.cpu())):
        with pytest.raises((ValueError, rl.RlkvError)):
            call(**bad)
