"""Chunks of new tokens over the paged cache: attention (rlkv_paged_chunk_attention) against the formula in 64 bits, ragged
writes (rlkv_paged_append_chunks) against single appends, bit for bit, rows read back (rlkv_paged_read) against what was
written, and the three together as a serving loop runs them.

Tolerances of attention.  With p the exact weights of a row and A = sum of p |v|: P is rounded to bf16 for the product, half a step
2^-8 of each weight, and the result once, 2^-8 of itself.  A score s is a sum of D products in fp32, off by at most
(D + 4) 2^-24 of sum |q k| / sqrt(D) -- which is below 2^-24 * 8 * max |s| + 2^-17 for standard normal rows of at most 128
elements: |q||k| / sqrt(D) < 25 --, the distance term and the cap by 2^-22 of their magnitudes, and a weight by as much of itself,
twice (numerator and sum): 2^-14 A covers them at the magnitudes here, and the exponentials' 2^-22.  lse: the same 2^-15 and its
own rounding, 2^-22 of its magnitude (and of the largest score's)."""
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


def scales(Hkv, fp8):
    return ([0.01 + 0.003 * h for h in range(Hkv)], [0.02 + 0.001 * h for h in range(Hkv)]) if fp8 else (None, None)


def make(hz, dev, Hkv, Hq, D, mask, S, W, lens, room, fp8, layers=1, spare=0):
    top = max(x + room for x in lens)
    pages = sum((x + room + 63) // 64 for x in lens) + spare
    ks, vs = scales(Hkv * layers, fp8)
    return hz.PagedCache(layers, Hkv, Hq, D, len(lens), pages, top, [int(c) for c in mask] * layers, S, W, device=dev, k_scale=ks, v_scale=vs)


def fill(cache, lens, Hkv, D, seed, dev, layer=0):
    """Opens and fills sequences; returns slots and the K and V rows they were given."""
    slots, rows = [], []
    for i, n in enumerate(lens):
        slots.append(cache.open_seq())
        k, v = rand_bf16((n, Hkv, D), seed + 2 * i).to(dev), rand_bf16((n, Hkv, D), seed + 2 * i + 1).to(dev)
        if n:
            cache.prefill(layer, slots[-1], k, v)
        rows.append((k, v))
    return slots, rows


def as_held(x, fp8, Hkv, which):
    """The values that a cache holds of rows x."""
    if not fp8:
        return x.double()
    s = torch.tensor(scales(Hkv, True)[which], dtype=torch.float32, device=x.device)[:, None]
    return (x.float() * (1 / s)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s.double()


def reference(q, rows, new, lens, counts, mask, S, W, cap, slopes, fp8):
    """out, A (per element sum of p |v|), lse and the largest |score| seen, in 64 bits."""
    Hq, D = q.shape[1:]
    Hkv = len(mask)
    G = Hq // Hkv
    outs, sizes, lses, tops = [], [], [], []
    at = 0
    for (k0, v0), n, m in zip(rows, lens, counts):
        if m == 0:
            continue
        kk = torch.cat([as_held(k0, fp8, Hkv, 0), new[0][at:at + m].double()])
        vv = torch.cat([as_held(v0, fp8, Hkv, 1), new[1][at:at + m].double()])
        key, pos = torch.arange(n + m, device=q.device), n + torch.arange(m, device=q.device)[:, None]
        x = torch.einsum("ihgd,jhd->hgij", q[at:at + m].double().view(m, Hkv, G, D), kk) / D ** 0.5
        if cap:
            x = cap * torch.tanh(x / cap)
        if slopes is not None:
            x = x - torch.tensor(slopes, dtype=torch.float64, device=q.device).view(Hkv, G, 1, 1) * (pos - key)
        full = torch.tensor([c == "1" for c in mask], device=q.device).view(Hkv, 1, 1, 1)
        seen = (key <= pos) & (full | (key < S) | (key > pos - W))
        tops.append(x.abs().masked_fill(~seen, 0).amax(-1).permute(2, 0, 1).reshape(m, Hq))
        x = x.masked_fill(~seen, -float("inf"))
        p = torch.softmax(x, -1)
        lses.append(torch.logsumexp(x, -1).permute(2, 0, 1).reshape(m, Hq))
        outs.append(torch.einsum("hgij,jhd->ihgd", p, vv).reshape(m, Hq, D))
        sizes.append(torch.einsum("hgij,jhd->ihgd", p, vv.abs()).reshape(m, Hq, D))
        at += m
    return tuple(torch.cat(x) for x in (outs, sizes, lses, tops))


def compare(out, lse, want):
    ref, size, ref_lse, top = want
    err = (out.double() - ref).abs()
    bound = (2.0 ** -8 + 2.0 ** -14) * size + 2.0 ** -8 * ref.abs() + 1e-6
    assert bool((err <= bound).all()), float((err / bound).max())
    err = (lse.double() - ref_lse).abs()
    bound = 2.0 ** -15 + 2.0 ** -22 * (ref_lse.abs() + top)
    assert bool((err <= bound).all()), float((err / bound).max())


CASES = [
    # Hkv, Hq, D, mask, sink, window, lens, counts, cap, slopes, fp8
    (1, 1, 64, "1", 0, 5, [0], [1], 0, False, False),
    (1, 4, 128, "1", 4, 60, [1], [1], 0, False, False),
    (2, 8, 64, "10", 4, 60, [63, 64, 65, 0], [1, 1, 1, 1], 0, False, False),
    (2, 8, 128, "10", 16, 112, [127, 128, 129, 0], [5, 1, 8, 3], 50.0, True, False),
    (8, 32, 128, "11011011", 16, 112, [3000], [5], 0, False, False),               # one long sequence, few rows
    (8, 32, 128, "11111111", 16, 112, [9000], [1], 0, True, False),
    (4, 28, 128, "1001", 16, 112, [500, 0, 77, 200], [1, 0, 37, 18], 0, True, False),   # seven heads, an empty chunk
    (4, 28, 128, "0110", 16, 112, [300, 1, 128], [300, 2, 129], 30.0, False, False),
    (3, 24, 128, "010", 4, 60, [64, 900, 3], [16, 1, 200], 0, False, False),        # eight heads
    (2, 2, 128, "01", 0, 5, [3, 4, 5, 6, 200], [1, 2, 300, 9, 130], 0, True, False),     # rings of five rows
    (2, 8, 64, "00", 40, 25, [0, 10, 39, 40, 41, 64, 65, 66], [80, 60, 3, 2, 1, 30, 26, 70], 20.0, True, False),  # sinks that the chunk brings
    (2, 8, 64, "01", 100, 3000, [4000, 2000], [2, 100], 0, False, False),           # a ring of 49 tiles
    (1, 8, 128, "1", 4, 60, [0], [513], 0, False, False),                           # a prompt of its own
    (8, 32, 128, "10110111", 16, 112, [1000], [333], 50.0, False, False),
    (2, 6, 64, "10", 4, 60, [0, 250, 1000], [700, 1, 64], 0, True, False),
    (2, 8, 128, "10", 16, 112, [65, 0, 300], [4, 1, 1], 0, False, True),
    (8, 32, 128, "11011011", 16, 112, [3000, 17, 640, 64], [4, 4, 4, 4], 0, True, True),
    (4, 28, 128, "1010", 16, 112, [777, 129, 128], [300, 1, 64], 30.0, False, True),
    (2, 2, 128, "01", 0, 5, [63, 190], [129, 260], 0, False, True),
    (2, 16, 128, "00", 16, 240, [300, 200, 10], [100, 1, 300], 50.0, True, True),
]


def build(hz, dev, Hkv, Hq, D, mask, S, W, lens, counts, cap, biased, fp8, seed=100, room=0):
    cache = make(hz, dev, Hkv, Hq, D, mask, S, W, lens, max(room, max(counts)), fp8)
    slots, rows = fill(cache, lens, Hkv, D, seed, dev)
    slopes = [2.0 ** (-8.0 * (j + 1) / Hq) for j in range(Hq)] if biased else None
    if cap or biased:
        cache.set_scores(cap, slopes)
    x = rand_bf16((sum(counts), Hq + 2 * Hkv, D), seed + 50).to(dev)
    return cache, slots, rows, slopes, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


@pytest.mark.parametrize("Hkv,Hq,D,mask,S,W,lens,counts,cap,biased,fp8", CASES)
def test_attention(hz, cuda_device, Hkv, Hq, D, mask, S, W, lens, counts, cap, biased, fp8):
    cache, slots, rows, slopes, q, k, v = build(hz, cuda_device, Hkv, Hq, D, mask, S, W, lens, counts, cap, biased, fp8)
    before = [cache.export_head(0, s, h) for s in slots for h in range(Hkv)]
    out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
    assert cache.status() == 0
    compare(out, lse, reference(q, rows, (k, v), lens, counts, mask, S, W, cap, slopes, fp8))
    again, lse2 = cache.attend_chunks(0, slots, counts, q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(out, again) and torch.equal(lse, lse2)     # the same bits, whatever the strides
    for a, b in zip(before, [cache.export_head(0, s, h) for s in slots for h in range(Hkv)]):
        for x, y in zip(a, b):
            np.testing.assert_array_equal(x, y)                   # the cache is as it was
    assert [cache.length(0, s) for s in slots] == lens


LARGE = [
    # two tiles of rows at a time (see the plan): the last of them alone, one page in the last tile, rows that end inside a tile
    (2, 8, 32, 128, "11111111", 16, 112, [9000, 9001, 4033], [300, 64, 333], 0, False, False),
    (2, 8, 32, 128, "11011111", 16, 2000, [9984, 17, 13000], [300, 4, 329], 50.0, True, False),
    (2, 8, 56, 128, "11110111", 16, 112, [8000, 100, 17001], [200, 129, 150], 0, True, False),
    (2, 8, 8, 128, "11111111", 16, 112, [22000], [1200], 20.0, False, False),
    (2, 8, 32, 64, "11111110", 16, 2000, [20031, 17, 29000], [300, 4, 329], 50.0, True, False),
    (2, 8, 32, 128, "11011011", 16, 112, [3000, 17, 640], [900, 4, 333], 0, True, True),
    (2, 4, 28, 128, "1101", 16, 112, [4033, 64, 0], [700, 129, 1500], 20.0, False, True),
    (2, 8, 32, 128, "00000000", 16, 1000, [2000], [2999], 0, False, True),
    (2, 2, 8, 128, "10", 40, 2000, [1990, 0], [65, 33], 50.0, True, True),
    (2, 1, 1, 128, "1", 16, 112, [0], [129], 0, False, True),
    # one, over many units
    (1, 8, 32, 128, "11111111", 16, 112, [2500], [1500], 0, False, False),
    (1, 8, 32, 128, "11011011", 16, 112, [3000, 17, 640], [900, 4, 333], 50.0, True, False),
    (1, 4, 28, 128, "1101", 16, 112, [4000, 100, 0], [700, 129, 1500], 0, False, False),
    (1, 4, 16, 64, "1111", 4, 60, [5000, 63], [1031, 800], 20.0, True, False),
    (1, 8, 32, 128, "01000010", 40, 2000, [1990, 0], [1500, 700], 0, True, False),
    (1, 4, 16, 128, "1011", 16, 112, [700] * 9, [130] + [1] * 8, 0, True, True),
    # many ranges in one unit, for each way of joining them
    (1, 1, 8, 128, "1", 16, 112, [30000], [17], 0, False, False),
    (2, 1, 8, 128, "1", 16, 112, [30001], [33], 50.0, False, True),
    (1, 2, 14, 64, "11", 16, 112, [12000], [40], 0, False, False),
    (0, 1, 8, 128, "1", 16, 112, [30000], [4], 0, False, False),
    (0, 1, 7, 128, "1", 16, 112, [29999], [3], 0, False, True),
]


@pytest.mark.parametrize("shape,Hkv,Hq,D,mask,S,W,lens,counts,cap,biased,fp8", LARGE)
def test_attention_of_large_calls(hz, rl, cuda_device, shape, Hkv, Hq, D, mask, S, W, lens, counts, cap, biased, fp8):
    plan = lambda shape: rl.rlkv_debug_chunk_plan(lens, counts, mask.count("1"), mask.count("0"), Hq // Hkv, S, W, shape)  # noqa: E731
    if D == 128:
        np.testing.assert_array_equal(plan(-2 if fp8 else -1), plan(shape))
    cache, slots, rows, slopes, q, k, v = build(hz, cuda_device, Hkv, Hq, D, mask, S, W, lens, counts, cap, biased, fp8)
    out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
    assert cache.status() == 0
    starts = np.cumsum([0] + counts)
    for i, (a, b) in enumerate(zip(starts, starts[1:])):
        compare(out[a:b], lse[a:b], reference(q[a:b], rows[i:i + 1], (k[a:b], v[a:b]), lens[i:i + 1], counts[i:i + 1], mask, S, W, cap, slopes, fp8))
    again, lse2 = cache.attend_chunks(0, slots, counts, q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(out, again) and torch.equal(lse, lse2)


def test_many_sequences(hz, cuda_device):
    lens = [(i * 37) % 400 for i in range(200)]
    counts = [1 + (i * 7) % 5 if i % 9 else 0 for i in range(200)]
    counts[150] = 400
    for fp8 in (False, True):
        cache, slots, rows, slopes, q, k, v = build(hz, cuda_device, 4, 16, 128, "1010", 16, 112, lens, counts, 0, True, fp8)
        out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
        assert cache.status() == 0
        compare(out, lse, reference(q, rows, (k, v), lens, counts, "1010", 16, 112, 0, slopes, fp8))


@pytest.mark.parametrize("cap,biased", [(0, False), (0, True), (30.0, False)])
def test_small_and_large_chunks_on_an_8_bit_cache(hz, cuda_device, cap, biased):
    """Enough of both for a launch of each: the same results whatever their order, and whatever stands between them."""
    lens = [1750 + 3 * i for i in range(26)] + [900, 64, 300, 0]
    counts = [1 + i % 8 for i in range(26)] + [512, 0, 9, 33]
    order = [28, 0, 1, 26, 27] + list(range(2, 20)) + [29] + list(range(20, 26))
    lens, counts = [lens[i] for i in order], [counts[i] for i in order]
    mask = "110111"
    rows = [m * 4 <= 32 for m in counts]
    assert sum(n * 5 for n, r in zip(lens, rows) if r) >= 6 * 148 * 256 and sum(n * 5 * 16 for n, r in zip(lens, rows) if not r) >= 2 * 148 * 256
    cache, slots, held, slopes, q, k, v = build(hz, cuda_device, 6, 24, 128, mask, 16, 112, lens, counts, cap, biased, True)
    out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
    assert cache.status() == 0
    compare(out, lse, reference(q, held, (k, v), lens, counts, mask, 16, 112, cap, slopes, True))
    again, lse2 = cache.attend_chunks(0, slots, counts, q.contiguous(), k.contiguous(), v.contiguous())
    assert torch.equal(out, again) and torch.equal(lse, lse2)
    few = [i for i, m in enumerate(counts) if 0 < m <= 8]          # alone they go out in the launch they have here
    parts = [list(x.split(counts)) for x in (q, k, v, out, lse)]
    small = [torch.cat([x[i] for i in few]) for x in parts]
    alone, lse3 = cache.attend_chunks(0, [slots[i] for i in few], [counts[i] for i in few], *small[:3])
    assert torch.equal(alone, small[3]) and torch.equal(lse3, small[4])


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("counts", [[3, 1, 4], [200, 1, 90]])
@pytest.mark.parametrize("cap", [0.0, 20.0])
def test_rows_of_others_have_no_effect(hz, rl, cuda_device, fp8, counts, cap):
    """Recycled pages that hold NaN behind the sequences' tokens, another sequence whose rows are NaN, NaN behind the last chunk:
    the same bits as without."""
    dev, Hkv, Hq, D, lens = cuda_device, 2, 8, 128, [70, 300, 129]
    total = sum(counts)

    def run(poison):
        cache = make(hz, dev, Hkv, Hq, D, "10", 16, 112, lens, 512, fp8)
        cache.set_scores(cap)
        old = [cache.open_seq() for _ in lens]     # fills every page and ring, then leaves
        for s in old:
            x = torch.full((512, Hkv, D), float("nan") if poison else 0.0, dtype=torch.bfloat16, device=dev)
            cache.prefill(0, s, x, x)
        for s in old:
            cache.close_seq(s)
        slots, rows = fill(cache, lens, Hkv, D, 7, dev)
        x = rand_bf16((total + 140, Hq + 2 * Hkv, D), 8).to(dev)
        x[total:] = float("nan") if poison else 0.0
        a = counts[0]
        x[a:a + counts[1]] = float("nan") if poison else 1.0
        out = torch.full((total + 140, Hq, D), 7.0, dtype=torch.bfloat16, device=dev)
        lse = torch.full((total + 140, Hq), 7.0, device=dev)
        rl.rlkv_paged_chunk_attention(cache.handle, 0, slots, counts, x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:], out, lse)
        assert cache.status() == 0
        assert bool((out[total:] == 7).all()) and bool((lse[total:] == 7).all())   # nothing behind the last chunk
        return [torch.cat([y[:a], y[a + counts[1]:total]]) for y in (out, lse)]

    for x, y in zip(run(False), run(True)):
        assert torch.equal(x, y)


def test_rows_do_not_depend_on_lse_or_order(hz, rl, cuda_device):
    """Without lse the same out; sequences given in another order get the same results to rounding (their ranges differ)."""
    lens, counts = [500, 65, 1200], [9, 40, 1]
    cache, slots, rows, _, q, k, v = build(hz, cuda_device, 2, 8, 128, "10", 16, 112, lens, counts, 0, False, False)
    out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
    alone = torch.empty_like(out)
    rl.rlkv_paged_chunk_attention(cache.handle, 0, slots, counts, q, k, v, alone)
    assert torch.equal(out, alone)
    parts = list(zip(*(x.split(counts) for x in (q, k, v))))
    turned = [torch.cat(x) for x in zip(*(parts[i] for i in (2, 0, 1)))]
    got, got_lse = cache.attend_chunks(0, [slots[i] for i in (2, 0, 1)], [counts[i] for i in (2, 0, 1)], *turned)
    compare(got, got_lse, reference(turned[0], [rows[i] for i in (2, 0, 1)], turned[1:], [1200, 500, 65], [1, 9, 40], "10", 16, 112, 0, None, False))


@pytest.mark.parametrize("counts", [[3, 2], [150, 3]])
@pytest.mark.parametrize("k_scale", [1e-12, 1e-36])
def test_queries_of_zeros_over_tiny_codes(hz, cuda_device, counts, k_scale):
    """An 8-bit cache whose scale times the queries' own leaves fp32: a query of zeros weighs every key that it sees the same."""
    dev, Hkv, Hq, D, lens = cuda_device, 2, 8, 128, [70, 20]
    cache = hz.PagedCache(1, Hkv, Hq, D, 2, 8, 256, [1, 0], 16, 112, device=dev, k_scale=[k_scale] * 2, v_scale=scales(Hkv, True)[1])
    slots, rows = fill(cache, lens, Hkv, D, 3, dev)
    x = rand_bf16((sum(counts), Hq + 2 * Hkv, D), 4).to(dev)
    q = torch.zeros_like(x[:, :Hq].contiguous())
    out, lse = cache.attend_chunks(0, slots, counts, q, x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
    assert cache.status() == 0
    compare(out, lse, reference(q, rows, (x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]), lens, counts, "10", 16, 112, 0, None, True))


WRITES = [
    # Hkv, D, mask, sink, window, fp8, lengths, then counts call by call
    (2, 64, "10", 4, 60, False, [[1, 63, 64, 65, 0], [64, 1, 0, 200, 3], [130, 130, 130, 1, 1]]),
    (2, 128, "01", 0, 5, False, [[3, 4], [1, 7], [300, 2]]),
    (3, 128, "010", 16, 112, True, [[10, 130, 64], [1, 1, 1], [5, 60, 129], [250, 0, 40]]),
    (2, 128, "10", 40, 25, True, [[20, 66], [21, 1], [30, 30], [17, 64]]),
    (1, 128, "0", 100, 300, True, [[90], [50], [700], [16]]),
    (1, 128, "1", 16, 112, False, [[40000], [100]]),
    (2, 64, "11", 16, 112, False, [[20000, 20000, 20000, 20000], [7, 8, 9, 10]]),   # more pages than one launch names
]


@pytest.mark.parametrize("Hkv,D,mask,S,W,fp8,calls", WRITES)
def test_append_chunks_are_single_appends(hz, cuda_device, Hkv, D, mask, S, W, fp8, calls):
    """Against rlkv_paged_prefill, which is single appends, and against rlkv_paged_append for the last tokens."""
    dev, n = cuda_device, len(calls[0])
    lens = [sum(c[i] for c in calls) for i in range(n)]
    cache, plain = (make(hz, dev, Hkv, Hkv, D, mask, S, W, lens, 8, fp8) for _ in range(2))
    a, b = [cache.open_seq() for _ in range(n)], [plain.open_seq() for _ in range(n)]
    for c, counts in enumerate(calls):
        x = rand_bf16((sum(counts), 2 * Hkv + 1, D), 60 + c).to(dev)
        k, v = x[:, :Hkv], x[:, Hkv + 1:]
        cache.append_chunks(0, a, counts, k, v)
        at = 0
        for i, m in enumerate(counts):
            if m:
                plain.prefill(0, b[i], k[at:at + m].contiguous(), v[at:at + m].contiguous())
            at += m
        assert [cache.length(0, s) for s in a] == [plain.length(0, s) for s in b]
    for step in range(5):
        k, v = rand_bf16((n, Hkv, D), 90 + step).to(dev), rand_bf16((n, Hkv, D), 190 + step).to(dev)
        cache.append_chunks(0, a[::-1], [1] * n, k.flip(0), v.flip(0))
        plain.append(0, b, k, v)
    for s, t in zip(a, b):
        for h in range(Hkv):
            for x, y in zip(cache.export_head(0, s, h), plain.export_head(0, t, h)):
                np.testing.assert_array_equal(x, y)
    q = rand_bf16((n, Hkv, D), 5).to(dev)              # the device's page table too
    assert torch.equal(cache.decode(0, a, q), plain.decode(0, b, q))
    assert cache.status() == 0


def test_append_chunks_takes_pages_in_order_and_all_or_none(hz, rl, cuda_device):
    cache = hz.PagedCache(1, 2, 8, 64, 3, 5, 256, [1, 0], 4, 60, device=cuda_device)
    slots = [cache.open_seq() for _ in range(3)]
    x = rand_bf16((400, 2, 64), 1).to(cuda_device)
    cache.append_chunks(0, slots, [64, 65, 1], x, x)
    assert cache.pages() == (1, 5)
    with pytest.raises(rl.RlkvError) as e:           # two more pages where there is one
        cache.append_chunks(0, slots, [1, 63, 64], x, x)
    assert e.value.code == rl.RLKV_EFULL
    with pytest.raises(rl.RlkvError) as e:           # past max_seq_len
        cache.append_chunks(0, slots, [0, 0, 256], x, x)
    assert e.value.code == rl.RLKV_EFULL
    assert cache.pages() == (1, 5) and [cache.length(0, s) for s in slots] == [64, 65, 1]
    cache.append_chunks(0, slots, [0, 63, 63], x, x)
    assert cache.pages() == (1, 5)
    cache.append_chunks(0, slots, [0, 0, 0], x[:0], x[:0])
    assert [cache.length(0, s) for s in slots] == [64, 128, 64]


@pytest.mark.parametrize("Hkv,D,mask,S,W,fp8,lens,first,counts", [
    (2, 64, "10", 4, 60, False, [200, 64, 1, 130], [0, 0, 0, 63], [200, 64, 1, 2]),
    (2, 128, "01", 0, 5, False, [3, 300], [1, 290], [2, 9]),
    (3, 128, "010", 16, 112, True, [500, 129, 64, 10], [0, 65, 63, 10], [500, 64, 1, 0]),
    (2, 128, "00", 40, 25, True, [39, 66, 700], [0, 0, 20], [39, 66, 680]),
    (1, 128, "0", 100, 300, True, [1000], [50], [950])])
def test_read(hz, rl, cuda_device, Hkv, D, mask, S, W, fp8, lens, first, counts):
    dev = cuda_device
    cache = make(hz, dev, Hkv, Hkv, D, mask, S, W, lens, 0, fp8)
    slots, rows = fill(cache, lens, Hkv, D, 30, dev)
    total = sum(counts)
    k, v = (torch.full((total + 3, Hkv, D), 7.0, dtype=torch.bfloat16, device=dev) for _ in range(2))
    rl.rlkv_paged_read(cache.handle, 0, slots, first, counts, k, v)
    at = 0
    for (kk, vv), n, f, m in zip(rows, lens, first, counts):
        t = torch.arange(f, f + m, device=dev)
        gone = ((t >= S) & (t < n - W))[:, None, None] & torch.tensor([c == "0" for c in mask], device=dev)[:, None]
        for w, (got, x) in enumerate(((k, kk), (v, vv))):
            # value(code) * scale: the fp32 product is within half a step of bf16's last place of its rounding, as exact in 64 bits
            want = as_held(x[f:f + m], fp8, Hkv, w).masked_fill(gone, 0)
            assert bool(((got[at:at + m].double() - want).abs() <= 2.0 ** -8 * want.abs()).all())
            if not fp8:
                assert torch.equal(got[at:at + m], want.to(torch.bfloat16))
            assert bool((got[at:at + m][gone.expand(m, Hkv, D)] == 0).all())
        at += m
    assert bool((k[total:] == 7).all()) and bool((v[total:] == 7).all())
    for bad in (dict(f=[x + 1 for x in lens], m=[0] * len(lens)), dict(f=first, m=[x + 1 for x in lens]), dict(f=[-1] * len(lens), m=[0] * len(lens))):
        with pytest.raises(rl.RlkvError) as e:
            rl.rlkv_paged_read(cache.handle, 0, slots, bad["f"], bad["m"], 4096, 4096)
        assert e.value.code == rl.RLKV_EINVAL


@pytest.mark.parametrize("fp8", [False, True])
def test_what_was_read_goes_back_in(hz, cuda_device, fp8):
    dev, lens, Hkv, D = cuda_device, [700, 64, 129, 10], 3, 128
    cache = make(hz, dev, Hkv, 2 * Hkv, D, "101", 16, 112, lens, 8, fp8)
    slots, _ = fill(cache, lens, Hkv, D, 40, dev)
    held = [[cache.export_head(0, s, h) for h in range(Hkv)] for s in slots]
    k, v = cache.read(0, slots, [0] * 4, lens)
    for s in slots:
        cache.close_seq(s)
    back = [cache.open_seq() for _ in lens]
    cache.append_chunks(0, back, lens, k, v)
    for s, rows in zip(back, held):
        for h in range(Hkv):
            for x, y in zip(cache.export_head(0, s, h), rows[h]):
                np.testing.assert_array_equal(x, y)


@pytest.mark.parametrize("Hkv,Hq,D,mask,S,W,fp8,interleaved", [(2, 8, 128, "10", 16, 112, False, False), (4, 28, 128, "0101", 16, 112, True, False),
                                                              (2, 8, 64, "01", 4, 60, False, True)])
def test_prompts_in_pieces_beside_decoding(hz, cuda_device, Hkv, Hq, D, mask, S, W, fp8, interleaved):
    """The serving loop: norms and rotation, attention, append, chunk after chunk, on two layers; then a draft of which some tokens
    are accepted, and a single token.  Every result against the formula in 64 bits on the rows as they were given."""
    dev, lens, layers = cuda_device, [0, 40, 500], 2
    schedule = [[100, 1, 1], [29, 1, 1], [1, 130, 1], [300, 1, 17], [4, 4, 4]]
    cache = make(hz, dev, Hkv, Hq, D, mask, S, W, lens, 700, fp8, layers=layers)
    table = hz.rotary_table(2048, D, device=dev)
    cache.set_rotary(table, D, interleaved)
    g = torch.Generator(device=dev).manual_seed(3)
    qw, kw = (1 + 0.2 * torch.randn((layers, D), generator=g, device=dev) for _ in range(2))
    cache.set_norms(qw, kw, 1e-5)
    ks, vs = scales(Hkv * layers, True)
    slots, rows = None, []
    for layer in range(layers):
        held = []
        if slots is None:
            slots = [cache.open_seq() for _ in lens]
        for i, n in enumerate(lens):
            k, v = rand_bf16((n, Hkv, D), 1000 + 10 * layer + i).to(dev), rand_bf16((n, Hkv, D), 2000 + 10 * layer + i).to(dev)
            if n:
                cache.prefill(layer, slots[i], k, v)
            held.append([k, v])
        rows.append(held)
    now = list(lens)
    for step, counts in enumerate(schedule):
        accepted = [2, 0, 4] if step == len(schedule) - 1 else counts
        for layer in range(layers):
            x = rand_bf16((sum(counts), Hq + 2 * Hkv, D), 5000 + 10 * step + layer).to(dev)
            q, k, v = x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
            pos = torch.cat([n + torch.arange(m) for n, m in zip(now, counts)]).to(dev)
            q, k = cache.rotate_chunks(layer, slots, counts, q, k)
            check_rotated(q, x[:, :Hq], qw[layer], pos, D, interleaved)
            check_rotated(k, x[:, Hq:Hq + Hkv], kw[layer], pos, D, interleaved)
            out, lse = cache.attend_chunks(layer, slots, counts, q, k, v)
            shown = rows[layer]
            if fp8:  # (this layer's scales)
                shown = [[held8(y, s[layer * Hkv:(layer + 1) * Hkv]) for y, s in zip(kv, (ks, vs))] for kv in shown]
            compare(out, lse, reference(q, shown, (k, v), now, counts, mask, S, W, 0, None, False))
            starts = np.cumsum([0] + counts)
            keep = torch.cat([torch.arange(a, a + m) for a, m in zip(starts, accepted)]).to(dev)
            cache.append_chunks(layer, slots, accepted, k[keep], v[keep])
            for i, (a, m) in enumerate(zip(starts, accepted)):
                rows[layer][i] = [torch.cat([old, y[a:a + m]]) for old, y in zip(rows[layer][i], (k, v))]
        now = [n + m for n, m in zip(now, accepted)]
        assert all(cache.length(layer, s) == n for layer in range(layers) for s, n in zip(slots, now))
    # a chunk of one token is the decode step behind its append (the token's own K and V rows exact, in 16 bits)
    q, k, v = (rand_bf16((3, h, D), 77 + h).to(dev) for h in (Hq, Hkv, Hkv))
    out, _ = cache.attend_chunks(0, slots, [1, 1, 1], q, k, v)
    cache.append_chunks(0, slots, [1, 1, 1], k, v)
    if not fp8:
        # both round P to bf16 and `out` is rounded once more: half a step each of sum p |v|, and |v| < 5.5
        assert float((out.float() - cache.decode(0, slots, q)).abs().max()) <= (2 * 2.0 ** -8 + 2.0 ** -8) * 5.5
    assert cache.status() == 0


def held8(x, s):
    s = torch.tensor(s, dtype=torch.float32, device=x.device)[:, None]
    return (x.float() * (1 / s)).clamp(-448, 448).to(torch.float8_e4m3fn).double() * s.double()


def check_rotated(got, x, weight, pos, rot, interleaved, eps=1e-5):
    from test_gpu_rotary import rotate64
    y = x.double() / torch.sqrt(x.double().square().mean(-1, keepdim=True) + eps) * weight.double()
    want, size = rotate64(y, pos.cpu().numpy(), rot, interleaved)
    # fp32: the sum of 128 squares, the root (2 units in the last place), three products: 2^-21 of the magnitudes; bf16 once
    err = (got.double().cpu() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 2.0 ** -20 * size + 2.0 ** -133).all()), float(err.max())


def test_captured_and_on_another_stream(hz, rl, cuda_device):
    """A captured attention of a split call, replayed on new inputs between calls of other shapes that use the same scratch; and a
    call on a stream of its own."""
    dev = cuda_device
    lens, counts = [3000, 100], [3, 2]
    cache, slots, rows, _, q, k, v = build(hz, dev, 4, 16, 128, "1011", 16, 112, lens, counts, 0, False, False, room=150)
    q, k, v = (x.contiguous() for x in (q, k, v))
    out, lse = torch.empty(q.shape, dtype=torch.bfloat16, device=dev), torch.empty(q.shape[:2], device=dev)
    call = lambda: rl.rlkv_paged_chunk_attention(cache.handle, 0, slots, counts, q, k, v, out, lse)  # noqa: E731
    call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call()
    other = rand_bf16((300, 24, 128), 9).to(dev)
    for seed in range(3):
        for x in (q, k, v):
            x.copy_(rand_bf16(tuple(x.shape), 300 + seed).to(dev))
        cache.attend_chunks(0, slots, [150, 150], other[:, :16], other[:, 16:20], other[:, 20:])
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        got = out.clone(), lse.clone()
        compare(*got, reference(q, rows, (k, v), lens, counts, "1011", 16, 112, 0, None, False))
        call()
        torch.cuda.synchronize()
        assert torch.equal(out, got[0]) and torch.equal(lse, got[1])
    side = torch.cuda.Stream(dev)
    side.wait_stream(torch.cuda.current_stream(dev))
    out.zero_()
    torch.cuda.synchronize()
    rl.rlkv_paged_chunk_attention(cache.handle, 0, slots, counts, q, k, v, out, lse, stream=side)
    side.synchronize()
    assert torch.equal(out, got[0])


def test_refusals(hz, rl, cuda_device):
    dev = cuda_device
    cache = make(hz, dev, 2, 8, 64, "10", 4, 60, [100, 20], 28, False)
    slots, _ = fill(cache, [100, 20], 2, 64, 1, dev)
    q, k, out = rand_bf16((200, 8, 64), 1).to(dev), rand_bf16((200, 2, 64), 2).to(dev), torch.zeros((200, 8, 64), dtype=torch.bfloat16, device=dev)
    ok = dict(layer=0, slots=slots, counts=[2, 1], q=q, k=k, v=k, out=out)
    call = lambda **x: rl.rlkv_paged_chunk_attention(cache.handle, *{**ok, **x}.values())  # noqa: E731
    for code, bad in ((rl.RLKV_EINVAL, dict(layer=1)), (rl.RLKV_EINVAL, dict(slots=[slots[0]] * 2)), (rl.RLKV_EINVAL, dict(slots=[0, 9])),
                      (rl.RLKV_EINVAL, dict(counts=[-1, 1])), (rl.RLKV_EFULL, dict(counts=[29, 1])), (rl.RLKV_EINVAL, dict(q=q.data_ptr() + 2))):
        with pytest.raises(rl.RlkvError) as e:
            call(**bad)
        assert e.value.code == code, bad
    for bad in (dict(counts=[1]), dict(q=q.float()), dict(q=q[:2]), dict(k=q), dict(q=q.cpu()), dict(out=out[:2]), dict(q=q[:1].expand(200, 8, 64)),
                dict(out=out.float())):
        with pytest.raises((ValueError, rl.RlkvError)):
            call(**bad)
    with pytest.raises(rl.RlkvError):   # neither norms nor rotation set
        cache.rotate_chunks(0, slots, [2, 1], q, k)
    w = torch.ones((1, 64), device=dev)
    for bad in (lambda: cache.set_norms(w[0, :63], w), lambda: cache.set_norms(w.double(), w), lambda: cache.set_norms(w, w, 0.0),
                lambda: cache.set_norms(w, w, float("nan")), lambda: cache.set_norms(w, w, 2.0), lambda: cache.set_norms(w.cpu(), w),
                lambda: rl.rlkv_paged_set_norms(cache.handle, w.data_ptr() + 4, w)):
        with pytest.raises((ValueError, rl.RlkvError)):
            bad()
    table = hz.rotary_table(101, 64, device=dev)
    cache.set_rotary(table, 64)
    with pytest.raises(rl.RlkvError) as e:   # a token past the table
        cache.rotate_chunks(0, slots, [2, 1], q, k)
    assert e.value.code == rl.RLKV_EINVAL
    cache.rotate_chunks(0, slots, [1, 8], q, k)
    call(counts=[0, 0])
    torch.cuda.synchronize()
    assert bool((out == 0).all())
