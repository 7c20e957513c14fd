"""Decode attention captured into CUDA graphs: a graph replayed any number of times, in any order with other graphs and with
calls outside of graphs on the same cache, gives the bits of the plain call.  Launches of more work items than CTAs hand their
items out at run time, so that what one launch leaves behind in the cache's counters is what the next one starts from."""
import numpy as np
import pytest
import torch

from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def hz(cuda_device):
    import paper_2510_08525_b200.harness as harness
    return harness


def interleave(calls, outs, want):
    """calls[i]() writes outs[i], whose bits have to be want[i]: captured, called plainly before the first replay, replayed alone
    and in turns, and called again."""
    graphs = []
    for call in calls:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            call()
        graphs.append(g)
    both = torch.cuda.CUDAGraph()
    with torch.cuda.graph(both):
        for call in calls:
            call()

    def check(run, which):
        for i in which:
            outs[i].zero_()
        run()
        torch.cuda.synchronize()
        for i in which:
            assert torch.equal(outs[i], want[i]), i

    every = range(len(calls))
    for i in every:
        check(calls[i], [i])                                       # captured, not replayed yet
    for _ in range(3):
        for i in every:
            check(graphs[i].replay, [i])
        check(both.replay, every)
        check(calls[0], [0])
    for i in reversed(every):
        check(graphs[i].replay, [i])
        check(calls[i], [i])
    check(both.replay, every)


@pytest.mark.parametrize("Hkv,Hq,D,mask,S,W,lens,fp8", [
    (8, 32, 128, "11011011", 16, 112, [9000, 8000, 64, 7000], False), (4, 28, 128, "1001", 16, 112, [20000, 300], True),
    (2, 8, 64, "10", 4, 60, [30000], False), (8, 8, 64, "00000000", 100, 3000, [4000] * 12, False)])
@pytest.mark.parametrize("cap,slope", [(0.0, 0.0), (20.0, 0.01)])
def test_paged_decode(hz, cuda_device, Hkv, Hq, D, mask, S, W, lens, fp8, cap, slope):
    dev, n = cuda_device, len(lens)
    scales = ([0.02] * Hkv, [0.03] * Hkv) if fp8 else (None, None)
    cache = hz.PagedCache(1, Hkv, Hq, D, n, sum(x // 64 + 2 for x in lens), max(lens) + 8, [int(c) for c in mask], S, W, device=dev,
                          k_scale=scales[0], v_scale=scales[1])
    slots = [cache.open_seq() for _ in lens]
    for s, x in zip(slots, lens):
        cache.prefill(0, s, rand_bf16((x, Hkv, D), 10 + s).to(dev), rand_bf16((x, Hkv, D), 90 + s).to(dev))
    cache.set_scores(cap, np.full(Hq, slope, np.float32) if slope else None)
    qs = [rand_bf16((n, Hq, D), 300 + i).to(dev) for i in range(3)]
    lists = [slots, slots[::-1], slots[:1]]                        # three calls of different batches
    qs = [q[:len(x)].contiguous() for q, x in zip(qs, lists)]
    want = [cache.decode(0, x, q).clone() for x, q in zip(lists, qs)]
    outs = [torch.empty_like(w) for w in want]
    interleave([lambda x=x, q=q, o=o: cache.decode(0, x, q, o) for x, q, o in zip(lists, qs, outs)], outs, want)
    assert cache.status() == 0


@pytest.mark.parametrize("mixed", [False, True])
def test_lock_step_decode(hz, cuda_device, mixed):
    dev, B, Hkv, Hq, D, n = cuda_device, 6, 4, 16, 128, 5000
    cache = hz.Cache(1, Hkv, Hq, D, B, n + 8, [1] * Hkv if mixed else [1, 0, 1, 1], 16, 112, device=dev)
    cache.prefill(0, rand_bf16((n, B, Hkv, D), 1).to(dev), rand_bf16((n, B, Hkv, D), 2).to(dev))
    alpha = torch.linspace(0.1, 0.9, Hkv, device=dev)
    run = (lambda q, o: cache.decode_mixed(0, q, alpha, o)) if mixed else (lambda q, o: cache.decode(0, q, o))
    qs = [rand_bf16((B, Hq, D), 5 + i).to(dev) for i in range(2)]
    want = [run(q, None).clone() for q in qs]
    outs = [torch.empty_like(w) for w in want]
    interleave([lambda q=q, o=o: run(q, o) for q, o in zip(qs, outs)], outs, want)
    assert cache.status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_whole_paged_step_with_scores(hz, cuda_device, fp8):
    """The captured step appends its token at the place it had at the capture, as often as it is replayed."""
    import paper_2510_08525_b200.binding as rl
    dev, L, Hkv, Hq, D, lens = cuda_device, 3, 4, 16, 128, [6000, 5000]
    n, mask = len(lens), [1, 0, 1, 1] * L
    scales = ([0.02] * (L * Hkv), [0.03] * (L * Hkv)) if fp8 else (None, None)
    caches = []
    for _ in range(2):
        c = hz.PagedCache(L, Hkv, Hq, D, n, 250, 6100, mask, 16, 112, device=dev, k_scale=scales[0], v_scale=scales[1])
        for i, x in enumerate(lens):
            c.open_seq()
            for l in range(L):
                c.prefill(l, i, rand_bf16((x, Hkv, D), 10 * i + l).to(dev), rand_bf16((x, Hkv, D), 700 + 10 * i + l).to(dev))
        c.set_scores(30.0, np.full(L * Hq, 0.02, np.float32))
        caches.append(c)
    k, v = rand_bf16((L, n, Hkv, D), 5).to(dev), rand_bf16((L, n, Hkv, D), 6).to(dev)
    q, q2 = rand_bf16((L, n, Hq, D), 7).to(dev), rand_bf16((n, Hq, D), 8).to(dev)
    want, out = torch.empty((L, n, Hq, D), device=dev), torch.empty((L, n, Hq, D), device=dev)
    rl.rlkv_paged_step(caches[0].handle, [0, 1], k, v, q, want)
    after = caches[0].decode(1, [0, 1], q2)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rl.rlkv_paged_step(caches[1].handle, [0, 1], k, v, q, out)
    for _ in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(caches[1].decode(1, [0, 1], q2), after)
    assert caches[0].status() == 0 and caches[1].status() == 0


@pytest.mark.parametrize("fp8", [False, True])
def test_rotated_append_and_decode_behind_it(hz, cuda_device, fp8):
    """A captured token goes where it belonged at the capture: on replays with other inputs its row is written anew, the rows before
    it and the sequences' lengths stay."""
    dev, Hkv, Hq, D, lens, mask = cuda_device, 4, 16, 128, [5000, 63, 6016], [1, 0, 1, 0]
    scales = ([0.02] * Hkv, [0.03] * Hkv) if fp8 else (None, None)
    table = hz.rotary_table(7000, D, device=dev)
    n, prompts, caches = len(lens), [], []
    for i, x in enumerate(lens):
        prompts.append([rand_bf16((x, Hkv, D), 10 * i + 1).to(dev), rand_bf16((x, Hkv, D), 10 * i + 2).to(dev)])
    for _ in range(4):
        c = hz.PagedCache(1, Hkv, Hq, D, n, 200, 6100, mask, 16, 112, device=dev, k_scale=scales[0], v_scale=scales[1])
        c.set_rotary(table, D)
        c.set_scores(20.0)
        for i, (k, v) in enumerate(prompts):
            c.open_seq()
            c.prefill(0, i, k, v)
        caches.append(c)
    tokens = [[rand_bf16((n, h, D), 50 + 3 * t + j).to(dev) for j, h in enumerate((Hq, Hkv, Hkv))] for t in range(3)]
    want = []
    for c, (q, k, v) in zip(caches[1:], tokens):
        qr = c.append_rotated(0, [0, 1, 2], q, k, v)
        want.append((qr.clone(), c.decode(0, [0, 1, 2], qr).clone()))
    import paper_2510_08525_b200.binding as rl
    c, given = caches[0], [x.clone() for x in tokens[0]]
    qr, out = torch.empty_like(given[0]), torch.empty((n, Hq, D), device=dev)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rl.rlkv_paged_append_rotated(c.handle, 0, [0, 1, 2], *given, qr)
        rl.rlkv_paged_decode_attention(c.handle, 0, [0, 1, 2], qr, out)
    for t in (0, 1, 2):
        for x, y in zip(given, tokens[t]):
            x.copy_(y)
        g.replay()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(qr, want[t][0]) and torch.equal(out, want[t][1])
    for i, x in enumerate(lens):
        assert c.length(0, i) == x + 1
        for h in range(Hkv):
            for a, b in zip(c.export_head(0, i, h), caches[3].export_head(0, i, h)):
                np.testing.assert_array_equal(a, b)
    assert c.status() == 0
