"""The launches of an attention call on chunks as it makes them (host arithmetic, no GPU): every chunk is in one of them, and in each every
key tile lies in one range, ranges of equal length by what a unit costs on that kind of cache."""
import random

import numpy as np
import pytest

from test_chunk_plan import binding, unit_tiles  # noqa: F401

COST = {(0, False): 5, (1, False): 4, (2, False): 3, (0, True): 10, (1, True): 4, (2, True): 3}   # key tiles of a unit's start and end


def all_launches(binding, *call):  # noqa: F811
    """Shape and ranges of each."""
    number = binding.rlkv_debug_chunk_launch(*call)[0]
    return [binding.rlkv_debug_chunk_launch(*call, which)[1:] for which in range(number)]


def check(binding, lens, counts, n_full, n_comp, group, sink, window, head_dim, fp8):  # noqa: F811
    launches = all_launches(binding, lens, counts, n_full, n_comp, group, sink, window, head_dim, fp8)
    small = [0 < m * group <= 32 for m in counts]
    assert len(launches) == 1 or (fp8 and len(launches) == 2 and launches[0][0] == 0 and any(small) and any(m * group > 32 for m in counts))
    for which, (shape, at) in enumerate(launches):
        mine = [m if m and (len(launches) == 1 or small[i] == (which == 0)) else 0 for i, m in enumerate(counts)]
        keys, tokens = ((64, 32 // group), (64, 128 // group), (128, 2 * (128 // group)))[shape]
        assert 1 <= len(at) - 1 <= (148 if shape == 2 else 296)
        assert shape or all(m <= tokens for m in mine)
        order, sizes = [], {}
        for i, (n, m) in enumerate(zip(lens, mine)):
            for j in range(-(-m // tokens)):
                for h in range(n_full + n_comp):
                    order.append((i, j, h))
                    sizes[i, j, h] = unit_tiles(n, m, j * tokens, tokens, keys, h < n_full, sink, window)
        cost = COST[shape, fp8]
        before, weight = 0, 0
        first, heavy = {}, {}
        for u in order:
            first[u], heavy[u] = before, weight
            before += sizes[u]
            weight += sizes[u] + cost
        end = (len(lens), 0, 0)
        first[end], heavy[end] = before, weight
        flat, share = [], weight // (len(at) - 1)
        for c, (i, j, h, t) in enumerate(at.tolist()):
            u = i, j, h
            assert t < sizes.get(u, 1)
            flat.append(first[u] + t)
            # an equal share of tiles and units' costs (a boundary inside a unit's cost lies at its start)
            want = weight * c // (len(at) - 1)
            assert heavy[u] <= want and want - heavy[u] == (t + cost if t else min(want - heavy[u], cost))
        assert flat[0] == 0 and flat[-1] == before and (np.diff(flat) >= 0).all()
        assert share >= 256 // keys or len(at) == 2
    return launches


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("lens,counts,n_full,n_comp,group,sink,window", [
    ([8192], [5], 6, 2, 4, 16, 112), ([8192], [700], 8, 0, 4, 16, 112), ([29999], [3], 1, 0, 7, 16, 112), ([1000], [1], 0, 1, 1, 0, 1),
    ([0, 3, 64, 65, 63, 200, 127, 128], [3, 0, 1, 65, 64, 1, 0, 130], 1, 3, 7, 16, 112), ([8064] * 32, [4] * 32, 6, 2, 4, 16, 112),
    ([10, 0, 0], [0, 300, 0], 0, 2, 8, 40, 25), ([2900] * 48, [512] + [1] * 47, 6, 2, 4, 16, 112), ([300] * 20, [40] * 20, 0, 8, 4, 16, 4080)])
def test_launches(binding, lens, counts, n_full, n_comp, group, sink, window, fp8):  # noqa: F811
    check(binding, lens, counts, n_full, n_comp, group, sink, window, 128, fp8)


def test_random_calls(binding):  # noqa: F811
    rng, two = random.Random(6), 0
    for _ in range(80):
        n, long, many = rng.randint(1, 60), rng.choice([500, 3000, 12000]), rng.random() < 0.5
        lens = [rng.randint(long // 2, long) if many else rng.choice([0, rng.randint(0, 400), rng.randint(0, long)]) for _ in range(n)]
        counts = [rng.choice([0, 1, 1, 1, rng.randint(1, 9), rng.randint(1, 700)]) for _ in range(n)]
        if not sum(counts):
            counts[0] = 1
        n_full, fp8 = rng.randint(0, 6), rng.random() < 0.7
        two += len(check(binding, lens, counts, n_full, rng.randint(0 if n_full else 1, 3), rng.randint(1, 8), rng.choice([0, 4, 16, 130]),
                         rng.choice([1, 60, 112, 300, 4000]), 128 if fp8 else rng.choice([64, 128]), fp8)) == 2
    assert two >= 5


@pytest.mark.parametrize("lens,counts", [([0] * 16, [240] * 16), ([60] * 201, [200] + [1] * 200), ([300] * 204, [200] * 4 + [1] * 200)])
def test_a_window_that_no_query_reaches_changes_no_launch(binding, lens, counts):  # noqa: F811
    for fp8 in (False, True):
        plans = [all_launches(binding, lens, counts, 2, 6, 4, 16, w, 128, fp8) for w in (500, 4080, 20000)]
        for other in plans[1:]:
            assert len(other) == len(plans[0])
            for (a, x), (b, y) in zip(plans[0], other):
                assert a == b
                np.testing.assert_array_equal(x, y)


def test_refusals(binding):  # noqa: F811
    b = binding
    ok = dict(lens=[10], counts=[1], n_full=1, n_comp=0, group=4, sink=0, window=1, head_dim=128, fp8=False)
    for bad in (dict(counts=[0]), dict(lens=[-1]), dict(counts=[-1]), dict(n_full=0), dict(group=9), dict(group=0), dict(window=0), dict(sink=-1),
                dict(head_dim=96), dict(head_dim=64, fp8=True), dict(counts=[(1 << 24) + 1])):
        with pytest.raises(b.RlkvError) as e:
            b.rlkv_debug_chunk_launch(**{**ok, **bad})
        assert e.value.code == b.RLKV_EINVAL
    with pytest.raises(ValueError):
        b.rlkv_debug_chunk_launch([1, 2], [1], 1, 0, 4, 0, 1)
    one, out, at = np.ones(1, np.int32).ctypes.data, b._ci(0), np.zeros((297, 4), np.int32).ctypes.data
    r = b.ctypes.byref(out)
    assert b.lib.rlkv_debug_chunk_launch(one, one, 1, 1, 0, 4, 0, 1, 128, 0, 1, r, r, r, at) == b.RLKV_EINVAL     # there is no second
    assert b.lib.rlkv_debug_chunk_launch(one, one, 1, 1, 0, 4, 0, 1, 128, 0, 0, r, r, r, 0) == b.RLKV_EINVAL
