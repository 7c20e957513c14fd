"""Attention of chunks where the queries' values are not those of a standard normal row: one channel far above the others, infinities
and NaN.

Tolerances.  An 8-bit cache takes the queries as two numbers, E4M3 and E5M2, at a power of two that brings a row's largest element to
128 .. 256.  Four bits go to the first; what is left has three or fewer while the element is 2^-13 of the largest or more, which E5M2
holds; below, the first is a multiple of 2^-9, and what it leaves, 2^-10 at most, is rounded to three bits, by 2^-14 at most: 2^-21 of the
largest element.  So a score is off by at most 2^-21 max |q| sum |k| / sqrt(D), and, as a sum of D products in fp32, by (D + 4) 2^-24 of
sum |q k| / sqrt(D).  lse is off by as much as its scores, by 2^-15 of the exponentials and their sum, and by its own rounding; a weight
relatively by twice as much (numerator and sum)."""
import pytest
import torch

from test_gpu_chunks import as_held, build, hz, reference  # noqa: F401
from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu

CHANNEL = 37


def with_channel(hz, dev, lens, counts, fp8, cached, own, mask="10", cap=0.0, seed=100):  # noqa: F811
    """As build, but every key holds the same number in one channel: `cached` those that the cache holds, `own` the chunks'."""
    Hkv, Hq, D, S, W = len(mask), 4 * len(mask), 128, 16, 112
    cache, slots, rows, _, q, k, v = build(hz, dev, Hkv, Hq, D, mask, S, W, [0] * len(lens), counts, cap, False, fp8, seed=seed, room=max(lens) + max(counts))
    rows = []
    for i, (s, n) in enumerate(zip(slots, lens)):
        kk, vv = rand_bf16((n, Hkv, D), seed + 2 * i).to(dev), rand_bf16((n, Hkv, D), seed + 2 * i + 1).to(dev)
        kk[..., CHANNEL] = cached
        if n:
            cache.prefill(0, s, kk, vv)
        rows.append((kk, vv))
    q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    k[..., CHANNEL] = own
    return cache, slots, rows, q, k, v


@pytest.mark.parametrize("factor", [300.0, 1000.0, -3000.0])
@pytest.mark.parametrize("lens,counts", [([5, 3, 70, 1], [3, 1, 4, 8]), ([5, 129], [300, 1]), ([64, 3], [33, 9])])
def test_queries_with_one_large_channel(hz, cuda_device, factor, lens, counts):  # noqa: F811
    """The channel is the same in all cached keys, so that it has no say in their weights; the chunk's own keys have it the other way round, so
    that the weights are those of the scores from the 8-bit codes."""
    sign = 1.0 if factor > 0 else -1.0
    cache, slots, rows, q, k, v = with_channel(hz, cuda_device, lens, counts, True, sign, -sign)
    q[..., CHANNEL] = factor
    out, lse = cache.attend_chunks(0, slots, counts, q, k, v)
    assert cache.status() == 0
    ref, size, ref_lse, top = reference(q, rows, (k, v), lens, counts, "10", 16, 112, 0, None, True)
    # sum |k| and sum |q k| of the largest key of each sequence
    big, both, at = torch.zeros_like(ref_lse), torch.zeros_like(ref_lse), 0
    for (kk, _), m in zip(rows, counts):
        held = as_held(kk, True, 2, 0).abs()
        rows_q = q[at:at + m].double().abs().view(m, 2, 4, 128)
        big[at:at + m] = held.sum(-1).amax(0).repeat_interleave(4)
        both[at:at + m] = torch.einsum("ihgd,jhd->ihgj", rows_q, held).amax(-1).reshape(m, 8)
        at += m
    score = (2.0 ** -21 * abs(factor) * big + 132 * 2.0 ** -24 * both) / 128 ** 0.5
    err = (lse.double() - ref_lse).abs()
    bound = score + 2.0 ** -15 + 2.0 ** -22 * (ref_lse.abs() + top)
    assert bool((err <= bound).all()), float((err / bound).max())
    err = (out.double() - ref).abs()
    bound = (2.0 ** -8 + 2.0 ** -14 + 2 * score[..., None]) * size + 2.0 ** -8 * ref.abs() + 1e-6
    assert bool((err <= bound).all()), float((err / bound).max())


BAD = [float("inf"), float("-inf"), float("nan")]


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,counts", [([40, 0], [3, 2]), ([9000, 17], [4, 1]), ([700, 5], [40, 3]), ([6000, 100], [300, 3])])
def test_queries_that_are_not_finite(hz, cuda_device, fp8, lens, counts):  # noqa: F811
    """An infinite or NaN query gives NaN, as the formula does, whether its keys lie in one piece or in many; the other rows do not change.
    (Every score of one sign of infinity: there is no largest that is finite, either.)"""
    cache, slots, rows, q, k, v = with_channel(hz, cuda_device, lens, counts, fp8, 1.0, 1.0)
    want, want_lse = cache.attend_chunks(0, slots, counts, q, k, v)
    for bad in BAD:
        for token, head in ((1, 0), (2, 7), (counts[0] - 1, 4)):
            x = q.clone()
            x[token, head, CHANNEL] = bad
            out, lse = cache.attend_chunks(0, slots, counts, x, k, v)
            assert cache.status() == 0
            assert bool(out[token, head].isnan().all()) and not bool(lse[token, head].isfinite())
            out[token, head], lse[token, head] = want[token, head], want_lse[token, head]
            assert torch.equal(out, want) and torch.equal(lse, want_lse)


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,counts", [([40, 0], [3, 2]), ([9000, 17], [4, 1]), ([700, 5], [40, 3])])
def test_infinite_queries_under_a_cap(hz, cuda_device, fp8, lens, counts):  # noqa: F811
    """A capped score of an infinite query is the cap: all keys weigh the same."""
    cache, slots, rows, q, k, v = with_channel(hz, cuda_device, lens, counts, fp8, 1.0, 1.0, cap=30.0)
    for bad in BAD[:2]:
        x = q.clone()
        x[2, 5, CHANNEL] = bad
        out, lse = cache.attend_chunks(0, slots, counts, x, k, v)
        assert cache.status() == 0
        ref, size, ref_lse, top = reference(x, rows, (k, v), lens, counts, "10", 16, 112, 30.0, None, fp8)
        err = (out.double() - ref).abs()
        assert bool((err <= (2.0 ** -8 + 2.0 ** -14) * size + 2.0 ** -8 * ref.abs() + 1e-6).all())
        assert bool(((lse.double() - ref_lse).abs() <= 2.0 ** -15 + 2.0 ** -22 * (ref_lse.abs() + top)).all())
