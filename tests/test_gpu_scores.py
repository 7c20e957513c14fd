"""Paged decode attention with capped and distance-biased scores (rlkv_paged_set_scores) against a plain softmax
in 64 bits over the tokens a head retains.

Tolerance: P is rounded to bf16 (8-bit cache: to f16) before the second product, half a step 2^-8 of each term,
so 2^-8 * sum p |v|; scores are fp32 -- 128 products accumulated in fp32 on |q.k| / sqrt(D) up to about 20, the cap
off by 2^-22 of itself, at most 1e-4 in the exponent for these inputs -- so another 2e-4 * sum p |v| with the sum's
own share; bf16 results are off by half a step of their own."""
import numpy as np
import pytest
import torch

from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def rl(cuda_device):
    import paper_2510_08525_b200.binding as binding
    return binding


@pytest.fixture(scope="module")
def hz(cuda_device):
    import paper_2510_08525_b200.harness as harness
    return harness


def reference(q, k, v, full, sink, window, cap, slopes):
    """q [Hq][D], k, v [n][Hkv][D] in 64 bits; returns the result and sum p |v|."""
    n, Hkv, D = k.shape
    G = q.shape[0] // Hkv
    t = torch.arange(n)
    out, size = torch.empty_like(q), torch.empty_like(q)
    for j in range(q.shape[0]):
        h = j // G
        keep = t if full[h] else t[(t < sink) | (t >= n - window)]
        x = k[keep, h] @ q[j] / np.sqrt(D)
        if cap:
            x = cap * torch.tanh(x / cap)
        if slopes is not None:
            x = x - float(slopes[j]) * (n - 1 - keep)
        p = torch.softmax(x, 0)
        out[j], size[j] = p @ v[keep, h], p @ v[keep, h].abs()
    return out, size


CASES = [
    # layers, Hkv, Hq, D, sink, window, mask, lengths, cap, slope base, fp8
    (1, 2, 8, 64, 4, 60, "10", [1, 63, 64, 65], 30.0, 0.5, False),
    (2, 2, 8, 64, 4, 12, "1001", [5, 200, 17, 129], 0.0, 0.3, False),
    (1, 4, 28, 128, 16, 112, "1001", [300, 1, 128, 1000, 77], 50.0, 0.0, False),
    (2, 8, 32, 128, 16, 112, "1101101100100001", [900, 64, 2500, 130], 5.0, 0.05, False),
    (1, 1, 8, 128, 0, 5, "0", [777, 3, 5, 6], 2.0, -0.2, False),
    (1, 2, 4, 128, 100, 200, "01", [1500, 299, 301, 50], 0.0, 1.0, True),
    (2, 4, 28, 128, 16, 112, "10010110", [400, 90, 1], 30.0, 0.1, True),
    (1, 1, 1, 128, 16, 48, "1", [40000], 20.0, 0.001, True),
]


@pytest.mark.parametrize("L,Hkv,Hq,D,S,W,mask,lens,cap,base,fp8", CASES)
def test_scored_decode(rl, hz, cuda_device, L, Hkv, Hq, D, S, W, mask, lens, cap, base, fp8):
    dev, mask = cuda_device, np.array([int(c) for c in mask]).reshape(L, Hkv)
    pages = sum((n + 1 + 63) // 64 for n in lens) + 1
    ks, vs = ([0.01 + 0.002 * i for i in range(L * Hkv)], [0.015 + 0.001 * i for i in range(L * Hkv)]) if fp8 else (None, None)
    cache = hz.PagedCache(L, Hkv, Hq, D, len(lens), pages, max(lens) + 1, mask, S, W, device=dev, k_scale=ks, v_scale=vs)
    slopes = (base * 2.0 ** -np.arange(L * Hq)).astype(np.float32) if base else None
    rows, slots = [], []
    for i, n in enumerate(lens):
        slots.append(cache.open_seq())
        per_layer = []
        for l in range(L):
            k, v = rand_bf16((n + 1, Hkv, D), 100 * i + l), rand_bf16((n + 1, Hkv, D), 7000 + 100 * i + l)
            cache.prefill(l, slots[i], k[:n].to(dev), v[:n].to(dev))
            per_layer.append((k, v))
        rows.append(per_layer)

    def held(x, scale, l):
        if not fp8:
            return x.double()
        s = torch.tensor(np.float32(scale[l * Hkv:(l + 1) * Hkv]))[:, None]
        return (x.float() * (1 / s)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s.double()

    def check(got, l, q, extra, bf16=False):
        for i, n in enumerate(lens):
            k, v = rows[i][l]
            n += extra
            want, size = reference(q[i].double(), held(k[:n], ks, l), held(v[:n], vs, l), mask[l], S, W, cap,
                                   None if slopes is None else slopes[l * Hq:(l + 1) * Hq])
            tol = (2.0 ** -8 + 2e-4) * size + (2.0 ** -8 * want.abs() if bf16 else 0)
            err = (got[i].double().cpu() - want).abs()
            assert bool((err <= tol).all()), (i, l, float((err / tol).max()))

    q = [rand_bf16((len(lens), Hq, D), 900 + l) for l in range(L)]
    plain = [cache.decode(l, slots, q[l].to(dev)) for l in range(L)]
    rl.rlkv_paged_set_scores(cache.handle, cap, slopes)
    for l in range(L):
        out = cache.decode(l, slots, q[l].to(dev))
        assert torch.equal(out, cache.decode(l, slots, q[l].to(dev)))          # the same call, the same bits
        check(out, l, q[l], 0)
        rl.rlkv_paged_set_output_bf16(cache.handle, 1)
        half = torch.empty((len(lens), Hq, D), dtype=torch.bfloat16, device=dev)
        rl.rlkv_paged_decode_attention(cache.handle, l, slots, q[l].to(dev), half)
        rl.rlkv_paged_set_output_bf16(cache.handle, 0)
        assert torch.equal(half, out.to(torch.bfloat16))
    # switched off again: the plain kernel's bits
    rl.rlkv_paged_set_scores(cache.handle, 0.0, np.zeros(L * Hq, np.float32))
    for l in range(L):
        assert torch.equal(cache.decode(l, slots, q[l].to(dev)), plain[l])
    # the whole step (every layer in one launch where there are several)
    rl.rlkv_paged_set_scores(cache.handle, cap, slopes)
    kk, vv = (torch.stack([torch.stack([rows[i][l][w][n] for i, n in enumerate(lens)]) for l in range(L)]).to(dev) for w in (0, 1))
    out = torch.empty((L, len(lens), Hq, D), device=dev)
    rl.rlkv_paged_step(cache.handle, slots, kk, vv, torch.stack(q).to(dev), out)
    for l in range(L):
        check(out[l], l, q[l], 1)
    assert cache.status() == 0


def test_large_products_stay_capped(rl, hz, cuda_device):
    """Products far past the cap: tanh saturates, every score is +-cap, nothing overflows."""
    dev = cuda_device
    cache = hz.PagedCache(1, 1, 4, 128, 1, 4, 256, [1], 4, 60, device=dev)
    s = cache.open_seq()
    k = rand_bf16((130, 1, 128), 1) * 100
    v = rand_bf16((130, 1, 128), 2)
    q = rand_bf16((1, 4, 128), 3) * 100
    cache.prefill(0, s, k.to(dev), v.to(dev))
    rl.rlkv_paged_set_scores(cache.handle, 3.0)
    got = cache.decode(0, [s], q.to(dev))
    want, size = reference(q[0].double(), k.double(), v.double(), [1], 4, 60, 3.0, None)
    # a product of 1e4 and more is off by up to 128 * 2^-24 of the sum of magnitudes (about 1e5 / sqrt(128)): 0.07
    # in x, times the slope of the cap, which is below 1e-3 wherever |x| > 4 * 3
    assert bool(((got[0].double().cpu() - want).abs() <= (2.0 ** -8 + 2e-3) * size).all())


def test_refusals(rl, hz, cuda_device):
    cache = hz.PagedCache(1, 2, 8, 128, 2, 8, 200, [1, 0], 4, 60, device=cuda_device)
    ok = np.full(8, 0.5, np.float32)
    for cap, slopes in ((-1.0, None), (float("nan"), None), (float("inf"), None), (1e-4, None), (1e7, None), (1001.0, None),
                        (0.0, np.full(8, np.nan, np.float32)), (0.0, np.full(8, np.inf, np.float32)), (0.0, np.full(8, -2e6, np.float32))):
        with pytest.raises(rl.RlkvError) as e:
            rl.rlkv_paged_set_scores(cache.handle, cap, slopes)
        assert e.value.code == rl.RLKV_EINVAL
    rl.rlkv_paged_set_scores(cache.handle, 1.0, ok)


def test_captured_call_reads_the_slopes_set_last(rl, hz, cuda_device):
    dev = cuda_device
    cache = hz.PagedCache(1, 2, 8, 128, 1, 8, 300, [1, 0], 4, 60, device=dev)
    s = cache.open_seq()
    cache.prefill(0, s, rand_bf16((200, 2, 128), 1).to(dev), rand_bf16((200, 2, 128), 2).to(dev))
    q, out = rand_bf16((1, 8, 128), 3).to(dev), torch.empty((1, 8, 128), device=dev)
    zeros, some, other = np.zeros(8, np.float32), np.full(8, 0.25, np.float32), np.linspace(0.1, 2, 8).astype(np.float32)
    cache.set_scores(20.0, some)
    cache.decode(0, [s], q, out)
    want = {}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        cache.decode(0, [s], q, out)
    for name, slopes in (("some", some), ("other", other), ("zeros", zeros), ("none", None), ("again", some)):
        cache.set_scores(20.0, slopes)
        want[name] = cache.decode(0, [s], q).clone()
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        # zeros: the launch without a distance term adds none, the captured one adds 0 * distance
        assert torch.equal(out, want[name]), name
    assert torch.equal(want["some"], want["again"]) and torch.equal(want["zeros"], want["none"])
    assert not torch.equal(want["some"], want["none"]) and not torch.equal(want["some"], want["other"])
