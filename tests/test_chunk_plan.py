"""How the work of an attention call on chunks is cut for the GPU's CTAs (host arithmetic, no GPU): every key tile of every
unit lies in exactly one range, ranges are of equal length, and the tiles are those that hold a visible key."""
import random

import numpy as np
import pytest


@pytest.fixture(scope="module")
def binding():
    from paper_2510_08525_b200 import build
    build.build()
    import paper_2510_08525_b200.binding as b
    return b


def unit_tiles(n, m, tok0, tokens, keys, full, sink, window):
    """Key tiles of a unit, from the visibility rule: the cache's rows (a ring as a whole while its window is seen), then the
    chunk's tiles that hold a key some query sees."""
    queries = np.arange(tok0, min(m, tok0 + tokens))
    if full:
        rows = n
    else:
        rows = min(n, sink + window) if n - 1 > n + tok0 - window else min(n, sink)
    tiles = set()
    for i in queries:
        j = np.arange(i + 1)
        if not full:
            j = j[(n + j < sink) | (j > i - window)]
        tiles.update(np.unique(j // keys).tolist())
    return -(-rows // keys) + len(tiles)


def check(binding, lens, counts, n_full, n_comp, group, sink, window, shape, ctas):
    at = binding.rlkv_debug_chunk_plan(lens, counts, n_full, n_comp, group, sink, window, shape, ctas)
    assert 1 <= len(at) - 1 <= ctas
    keys, tokens = ((64, 32 // group), (64, 128 // group), (128, 2 * (128 // group)))[shape]
    order, sizes = [], {}
    for i, (n, m) in enumerate(zip(lens, counts)):
        for j in range(-(-m // tokens)):
            for h in range(n_full + n_comp):
                order.append((i, j, h))
                sizes[i, j, h] = unit_tiles(n, m, j * tokens, tokens, keys, h < n_full, sink, window)
    first = {u: x for u, x in zip(order, np.cumsum([0] + [sizes[u] for u in order]))}
    total = sum(sizes.values())
    ends = {(len(lens), 0, 0): total}
    flat = []
    for i, j, h, t in at.tolist():
        assert (i, j, h) in ends or t < sizes[i, j, h]
        flat.append(ends.get((i, j, h), first.get((i, j, h))) + t)
    assert flat[0] == 0 and flat[-1] == total
    lengths = np.diff(flat)
    assert (lengths >= 0).all()
    # a unit counts some tiles more than it has: a range is at most an equal share of both
    share = (total + (5, 4, 3)[shape] * len(order)) / (len(at) - 1)
    assert lengths.max() <= share + 1


@pytest.mark.parametrize("shape", [0, 1, 2])
@pytest.mark.parametrize("lens,counts,n_full,n_comp,group,sink,window,ctas", [
    ([8192], [5], 6, 2, 4, 16, 112, 296), ([8192], [700], 8, 0, 4, 16, 112, 148), ([0], [1], 1, 0, 1, 0, 5, 296),
    ([0, 3, 64, 65, 63, 200, 127, 128], [3, 0, 1, 65, 64, 1, 0, 130], 1, 3, 7, 16, 112, 296),
    ([10, 0, 0], [0, 300, 0], 0, 2, 8, 40, 25, 17), ([5, 500, 129], [70, 200, 1], 0, 1, 3, 100, 60, 296), ([1000], [1], 0, 1, 1, 0, 1, 1)])
def test_ranges(binding, lens, counts, n_full, n_comp, group, sink, window, shape, ctas):
    check(binding, lens, counts, n_full, n_comp, group, sink, window, shape, ctas)


def test_random_batches(binding):
    rng = random.Random(5)
    for _ in range(60):
        n = rng.randint(1, 6)
        lens = [rng.choice([0, rng.randint(0, 400), rng.randint(0, 3000)]) for _ in range(n)]
        counts = [rng.choice([0, 1, rng.randint(1, 9), rng.randint(1, 300)]) for _ in range(n)]
        if not sum(counts):
            counts[0] = 1
        n_full = rng.randint(0, 3)
        check(binding, lens, counts, n_full, rng.randint(0 if n_full else 1, 3), rng.randint(1, 8), rng.choice([0, 4, 16, 130]),
              rng.choice([1, 5, 60, 112, 300]), rng.choice([0, 1, 2]), rng.choice([1, 7, 148, 296]))


def test_refusals(binding):
    for bad in (([1], [0], 1, 0, 4, 0, 1), ([-1], [1], 1, 0, 4, 0, 1), ([1], [-1], 1, 0, 4, 0, 1), ([1], [1], 0, 0, 4, 0, 1),
                ([1], [1], 1, 0, 9, 0, 1), ([1], [1], 1, 0, 4, 0, 0)):
        with pytest.raises(binding.RlkvError) as e:
            binding.rlkv_debug_chunk_plan(*bad)
        assert e.value.code == binding.RLKV_EINVAL
    with pytest.raises(binding.RlkvError):
        binding.rlkv_debug_chunk_plan([1], [1], 1, 0, 4, 0, 1, 1, 297)


@pytest.mark.parametrize("shape", [-1, -2])
@pytest.mark.parametrize("lens,counts", [([0] * 16, [240] * 16), ([0, 30, 5, 100], [700, 1, 90, 33]), ([100] * 40, [1] * 39 + [300])])
def test_a_window_that_no_query_reaches_changes_nothing(binding, lens, counts, shape):
    """A sequence is counted with the rows it has, not with those its rings have room for."""
    reach = max(n + m for n, m in zip(lens, counts))
    plans = [binding.rlkv_debug_chunk_plan(lens, counts, 2, 6, 4, 16, window, shape) for window in (reach, reach + 1, 4 * reach, 20000)]
    for plan in plans[1:]:
        np.testing.assert_array_equal(plans[0], plan)
