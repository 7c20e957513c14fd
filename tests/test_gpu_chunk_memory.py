"""The memory of attention on chunks: taken by the first call that attends some and by no other, or the caller's; and with any amount of it the
same results to rounding, nothing written behind it."""
import numpy as np
import pytest
import torch

from test_gpu_chunks import build, compare, hz, reference, rl, scales  # noqa: F401
from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu

HKV, HQ, D, MASK, S, W = 2, 8, 128, "10", 16, 112
# lengths and new tokens: 32 rows cut into many pieces and into few, 128 rows, two times 128 (or one, of an 8-bit cache), both beside one another
CALLS = [([30000, 5], [4, 4]), ([900, 300], [8, 1]), ([9000, 300], [17, 1]), ([12000, 0], [700, 129]), ([40, 3000], [333, 1])]


def in_a_buffer(rl, dev, fp8):  # noqa: F811
    """A function that makes a cache in a caller's buffer, and the buffer with a megabyte behind it that holds 0x5a."""
    shape = (1, HKV, HQ, D, 2, 1200, 32000, np.array([int(c) for c in MASK], np.uint8), S, W)
    size = (rl.rlkv_paged_size_fp8 if fp8 else rl.rlkv_paged_size)(*shape)
    buf = torch.full((size + 1024 + (1 << 20),), 0x5a, dtype=torch.uint8, device=dev)
    buf = buf[-buf.data_ptr() % 1024:]
    guard = buf[size:size + (1 << 20) - 1024]
    new = lambda: rl.rlkv_paged_create_fp8(*shape, *scales(HKV, True), buf, size) if fp8 else rl.rlkv_paged_create(*shape, buf, size)  # noqa: E731
    return new, guard


def attend(rl, hz, dev, handle, lens, counts, fp8):  # noqa: F811
    """Fills two sequences, attends their chunks, compares with the formula and closes them."""
    other, _, rows, _, q, k, v = build(hz, dev, HKV, HQ, D, MASK, S, W, lens, counts, 0, False, fp8)
    other.close()
    slots = [rl.rlkv_paged_seq_open(handle) for _ in lens]
    for s, (kk, vv) in zip(slots, rows):
        if len(kk):
            rl.rlkv_paged_prefill(handle, 0, s, kk, vv, len(kk))
    out, lse = torch.empty((sum(counts), HQ, D), dtype=torch.bfloat16, device=dev), torch.empty((sum(counts), HQ), device=dev)
    rl.rlkv_paged_chunk_attention(handle, 0, slots, counts, q, k, v, out, lse)
    compare(out, lse, reference(q, rows, (k, v), lens, counts, MASK, S, W, 0, None, fp8))
    for s in slots:
        rl.rlkv_paged_seq_close(handle, s)
    assert rl.rlkv_paged_kernel_status(handle) == 0
    return out, lse


@pytest.mark.parametrize("fp8", [False, True])
def test_memory_is_taken_by_the_first_call(hz, rl, cuda_device, fp8):  # noqa: F811
    dev = cuda_device
    new, guard = in_a_buffer(rl, dev, fp8)
    rl.rlkv_paged_destroy(new())    # (the kernels' code is loaded now)
    free = lambda: (torch.cuda.synchronize(), torch.cuda.mem_get_info()[0])[1]  # noqa: E731
    before = free()
    handle = new()
    slot = rl.rlkv_paged_seq_open(handle)
    x = rand_bf16((70, HKV, D), 1).to(dev)
    q, out = rand_bf16((1, HQ, D), 2).to(dev), torch.empty((1, HQ, D), device=dev)
    rl.rlkv_paged_append_chunks(handle, 0, [slot], [70], x, x)
    rl.rlkv_paged_decode_attention(handle, 0, [slot], q, out)
    torch.cuda.synchronize()
    assert free() >= before - (2 << 20)      # (torch's own 2 MB at most)
    rl.rlkv_paged_seq_close(handle, slot)
    size = rl.rlkv_paged_chunk_scratch_size(handle)
    assert size == 2 * 296 * 128 * (D + 2) * 4
    for lens, counts in CALLS:
        attend(rl, hz, dev, handle, lens, counts, fp8)
    torch.cuda.empty_cache()
    taken = free()
    rl.rlkv_paged_destroy(handle)
    assert size <= free() - taken <= size + (2 << 20)
    assert bool((guard == 0x5a).all())


@pytest.mark.parametrize("fp8", [False, True])
@pytest.mark.parametrize("ctas", [296, 100, 3, 1, 0])
def test_any_amount_of_memory_does(hz, rl, cuda_device, fp8, ctas):  # noqa: F811
    """The caller's memory, for this many CTAs of 128 rows (four times as many of 32, half as many of 256): the library takes none."""
    dev = cuda_device
    new, guard = in_a_buffer(rl, dev, fp8)
    handle = new()
    size = 2 * ctas * 128 * (D + 2) * 4
    scratch = torch.full((size + (1 << 20),), 0x5a, dtype=torch.uint8, device=dev)
    rl.rlkv_paged_set_chunk_scratch(handle, scratch, size)
    for lens, counts in CALLS:
        attend(rl, hz, dev, handle, lens, counts, fp8)
    assert bool((scratch[size:] == 0x5a).all()) and bool((guard == 0x5a).all())
    assert ctas < 296 or not bool((scratch[:size] == 0x5a).all())
    torch.cuda.empty_cache()
    torch.cuda.synchronize()
    free = torch.cuda.mem_get_info()[0]
    rl.rlkv_paged_destroy(handle)
    assert torch.cuda.mem_get_info()[0] == free


def test_the_first_call_may_be_a_captured_one(hz, rl, cuda_device):  # noqa: F811
    """And with the caller's memory, then without, the same bits."""
    dev, lens, counts = cuda_device, [9000, 300], [4, 1]
    cache, slots, rows, _, q, k, v = build(hz, dev, HKV, HQ, D, MASK, S, W, lens, counts, 0, False, False)
    q, k, v = (x.contiguous() for x in (q, k, v))
    out, lse = torch.zeros(q.shape, dtype=torch.bfloat16, device=dev), torch.zeros(q.shape[:2], device=dev)
    call = lambda: rl.rlkv_paged_chunk_attention(cache.handle, 0, slots, counts, q, k, v, out, lse)  # noqa: E731
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    graph.replay()
    torch.cuda.synchronize()
    compare(out, lse, reference(q, rows, (k, v), lens, counts, MASK, S, W, 0, None, False))
    want = out.clone(), lse.clone()
    for scratch in (torch.empty(rl.rlkv_paged_chunk_scratch_size(cache.handle), dtype=torch.uint8, device=dev), None):
        rl.rlkv_paged_set_chunk_scratch(cache.handle, scratch)
        for run in (call, graph.replay):
            out.zero_()
            run()
            torch.cuda.synchronize()
            assert torch.equal(out, want[0]) and torch.equal(lse, want[1])
    assert cache.status() == 0


def test_refusals(hz, rl, cuda_device):  # noqa: F811
    cache, *_ = build(hz, cuda_device, HKV, HQ, D, MASK, S, W, [40], [4], 0, False, False)
    x = torch.empty(4096, dtype=torch.uint8, device=cuda_device)
    for bad in (x[8:], x[::2], x.cpu(), torch.empty(4096, dtype=torch.uint8).pin_memory()):
        with pytest.raises((ValueError, rl.RlkvError)):
            rl.rlkv_paged_set_chunk_scratch(cache.handle, bad)
