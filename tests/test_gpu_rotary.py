"""Appending rotated keys to the paged cache (rlkv_rotary_table, rlkv_paged_append_rotated,
rlkv_paged_prefill_rotated) against a rotation in 64 bits, and against the plain append of the rotated rows,
whose cache bytes have to be the same.

Tolerances: a product pair a cos - b sin is computed in fp32 from exact bf16 inputs and a table off by half a
step of fp32 -- at most 4 * 2^-24 * (|a| + |b|) -- and rounded once, half a step of the result's type: 2^-8 of
the value in bf16, 2^-4 in E4M3 (2^-10 below its normal range, in units of the scale)."""
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


def inv_freq(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / rot)


def make_table(rl, rot, rows, dev):
    t = torch.empty((rows, rot // 2, 2), dtype=torch.float32, device=dev)
    rl.rlkv_rotary_table(inv_freq(rot), rows, t)
    return t


def rotate64(x, pos, rot, interleaved):
    """x [tokens][heads][D] in 64 bits; returns the rotated rows and |a| + |b| of every element's pair."""
    x = x.double().cpu()
    ang = torch.as_tensor(np.asarray(pos, np.float64)[:, None] * inv_freq(rot))[:, None]
    i = (np.arange(0, rot, 2), np.arange(1, rot, 2)) if interleaved else (np.arange(rot // 2), np.arange(rot // 2) + rot // 2)
    a, b = x[..., i[0]], x[..., i[1]]
    out, size = x.clone(), torch.zeros_like(x)
    out[..., i[0]] = a * ang.cos() - b * ang.sin()
    out[..., i[1]] = b * ang.cos() + a * ang.sin()
    size[..., i[0]] = size[..., i[1]] = a.abs() + b.abs()
    return out, size


def check_bf16(got, want, size):
    err = (got.double().cpu() - want).abs()
    assert bool((err <= 2.0 ** -8 * want.abs() + 4 * 2.0 ** -24 * size + 2.0 ** -133).all()), float(err.max())


def test_rotary_table_is_exact_at_far_positions(rl, cuda_device):
    rows, rot = 65536, 128
    t = make_table(rl, rot, rows, cuda_device).double().cpu()
    pos = np.concatenate([np.arange(100), np.arange(rows - 100, rows), np.arange(0, rows, 997)])
    ang = torch.as_tensor(pos[:, None] * inv_freq(rot))
    # half a step of fp32 below 1, and the 64-bit argument's own rounding (2^-53 of 65536)
    assert float((t[pos, :, 0] - ang.cos()).abs().max()) <= 2.0 ** -25 + 1e-11
    assert float((t[pos, :, 1] - ang.sin()).abs().max()) <= 2.0 ** -25 + 1e-11


def fused(n, Hq, Hkv, D, seed, dev):
    """q, k, v as slices of one projection's output."""
    x = rand_bf16((n, Hq + 2 * Hkv, D), seed).to(dev)
    return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]


def apart(n, Hq, Hkv, D, seed, dev):
    return tuple(x.contiguous() for x in fused(n, Hq, Hkv, D, seed, dev))


def same_state(a, b, slot_a, slot_b, layer=0):
    for h in range(a.kv_heads):
        for x, y in zip(a.export_head(layer, slot_a, h), b.export_head(layer, slot_b, h)):
            np.testing.assert_array_equal(x, y)


CASES = [
    # Hkv, Hq, D, sink, window, mask, rot, interleaved, sliced, fp8, prompt lengths
    (2, 8, 64, 4, 60, "10", 64, False, False, False, [1, 63, 65]),
    (2, 2, 64, 0, 5, "01", 32, True, True, False, [7, 200]),
    (4, 28, 128, 16, 112, "1001", 128, False, True, False, [300, 1, 64]),
    (4, 28, 128, 16, 112, "0110", 64, False, False, True, [129, 700]),
    (3, 24, 128, 4, 60, "010", 128, True, True, True, [64, 65, 3]),
    (1, 8, 128, 16, 48, "1", 16, False, False, False, [40000]),       # two launches
    (1, 1, 128, 16, 48, "0", 112, True, True, True, [33000]),
]


@pytest.mark.parametrize("Hkv,Hq,D,S,W,mask,rot,interleaved,sliced,fp8,lens", CASES)
def test_rotated_prefill_and_append(rl, hz, cuda_device, Hkv, Hq, D, S, W, mask, rot, interleaved, sliced, fp8, lens):
    dev, mask = cuda_device, [int(c) for c in mask]
    max_len, pages = max(lens) + 80, sum((n + 80 + 63) // 64 for n in lens)
    scales = ([0.01 + 0.003 * h for h in range(Hkv)], [0.02 + 0.001 * h for h in range(Hkv)]) if fp8 else (None, None)
    make = lambda: hz.PagedCache(1, Hkv, Hq, D, len(lens), pages, max_len, mask, S, W, device=dev, k_scale=scales[0], v_scale=scales[1])  # noqa: E731
    cache, plain = make(), make()
    table = make_table(rl, rot, max_len, dev)
    rl.rlkv_paged_set_rotary(cache.handle, table, max_len, rot, interleaved)
    give = fused if sliced else apart
    slots = []
    for i, n in enumerate(lens):
        q, k, v = give(n, Hq, Hkv, D, 10 + i, dev)
        a, b = cache.open_seq(), plain.open_seq()
        slots.append((a, b))
        q_out = torch.full((n + 1, Hq, D), 7.0, dtype=torch.bfloat16, device=dev)
        k_out = torch.full((n + 1, Hkv, D), 7.0, dtype=torch.bfloat16, device=dev)
        rl.rlkv_paged_prefill_rotated(cache.handle, 0, a, q, k, v, n, q_out, k_out)
        check_bf16(q_out[:n], *rotate64(q, np.arange(n), rot, interleaved))
        want, size = rotate64(k, np.arange(n), rot, interleaved)
        check_bf16(k_out[:n], want, size)
        assert bool((q_out[n] == 7).all()) and bool((k_out[n] == 7).all())      # nothing behind the last token
        plain.prefill(0, b, k_out[:n].contiguous(), v.contiguous())
        if not fp8:
            same_state(cache, plain, a, b)
        else:
            check_codes(cache, plain, a, b, want, size, scales[0], S, W)
    # 70 single tokens each: page borders and ring wraps, some appended without queries, one call in place
    for step in range(70):
        q, k, v = give(len(lens), Hq, Hkv, D, 1000 + step, dev)
        pos = [n + step for n in lens]
        want, size = rotate64(k, pos, rot, interleaved)
        out = torch.empty((len(lens), Hq, D), dtype=torch.bfloat16, device=dev)
        if step == 5:
            rl.rlkv_paged_append_rotated(cache.handle, 0, [a for a, _ in slots], None, k, v, None)
        else:
            inp = q.contiguous() if step == 6 else q
            before = inp.clone()
            out = inp if step == 6 else out
            rl.rlkv_paged_append_rotated(cache.handle, 0, [a for a, _ in slots], inp, k, v, out)
            check_bf16(out, *rotate64(before, pos, rot, interleaved))
        # the rotated rows, rounded as the library rounds them, go into the other cache
        plain.append(0, [b for _, b in slots], round_like(rl, hz, k, pos, rot, interleaved, table), v.contiguous())
    for a, b in slots:
        if not fp8:
            same_state(cache, plain, a, b)
    assert cache.status() == 0
    for (a, _), n in zip(slots, lens):
        assert cache.length(0, a) == n + 70


def round_like(rl, hz, k, pos, rot, interleaved, table):
    """The fp32 rotation on the GPU with one fused multiply-add per product pair, rounded to bf16."""
    x = k.float()
    f = table[torch.as_tensor(pos, device=k.device)][:, None].double()
    cos, sin = f[..., 0], f[..., 1]
    i = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., i[0]].double(), x[..., i[1]].double()
    # fma(a, cos, -(b sin rounded)): the product in 64 bits is exact, one rounding each
    y = x.clone()
    y[..., i[0]] = (a * cos - (b * sin).float().double()).float()
    y[..., i[1]] = (b * cos + (a * sin).float().double()).float()
    return y.to(torch.bfloat16)


def check_codes(cache, plain, a, b, want, size, k_scale, S, W):
    for h in range(cache.kv_heads):
        gk, gv, gt = cache.export_head(0, a, h)
        _, pv, pt = plain.export_head(0, b, h)
        np.testing.assert_array_equal(gt, pt)
        np.testing.assert_array_equal(gv, pv)                       # V passes through untouched
        held = gt >= 0
        x = torch.from_numpy(gk.astype(np.uint8)[held]).view(torch.float8_e4m3fn).double()
        w = (want[gt[held], h] / k_scale[h]).clamp(-448, 448)
        tol = 2.0 ** -4 * w.abs() + 2.0 ** -10 + 8 * 2.0 ** -24 * size[gt[held], h] / k_scale[h]
        assert bool(((x - w).abs() <= tol).all())


@pytest.mark.parametrize("Hkv,Hq,S,W,mask,rot,interleaved,sliced,lens", [
    (4, 28, 16, 112, "0110", 64, False, False, [129, 700, 1]), (3, 24, 4, 60, "010", 128, True, True, [64, 65, 3]),
    (2, 2, 0, 5, "10", 112, False, True, [60, 127]), (1, 8, 100, 200, "0", 16, True, False, [250])])
def test_single_tokens_in_8_bits(rl, hz, cuda_device, Hkv, Hq, S, W, mask, rot, interleaved, sliced, lens):
    """The codes of 140 tokens appended one by one behind prompts: K codes of the fp32 rotation, V codes those of the plain append,
    across page borders, over ring wraps, on sequences at different places of their pages."""
    dev, mask, more, D = cuda_device, [int(c) for c in mask], 140, 128
    max_len, pages = max(lens) + more, sum((n + more + 63) // 64 for n in lens)
    k_scale, v_scale = [0.01 + 0.003 * h for h in range(Hkv)], [0.02 + 0.001 * h for h in range(Hkv)]
    make = lambda: hz.PagedCache(1, Hkv, Hq, D, len(lens), pages, max_len, mask, S, W, device=dev, k_scale=k_scale, v_scale=v_scale)  # noqa: E731
    cache, plain = make(), make()
    rl.rlkv_paged_set_rotary(cache.handle, make_table(rl, rot, max_len, dev), max_len, rot, interleaved)
    give = fused if sliced else apart
    slots, history = [], []
    for i, n in enumerate(lens):
        _, k, v = give(n, Hq, Hkv, D, 10 + i, dev)
        a, b = cache.open_seq(), plain.open_seq()
        slots.append((a, b))
        rl.rlkv_paged_prefill_rotated(cache.handle, 0, a, None, k, v, n, None)
        plain.prefill(0, b, k.contiguous(), v.contiguous())
        history.append([rotate64(k, np.arange(n), rot, interleaved)])
    for step in range(more):
        q, k, v = give(len(lens), Hq, Hkv, D, 1000 + step, dev)
        out = torch.empty((len(lens), Hq, D), dtype=torch.bfloat16, device=dev)
        rl.rlkv_paged_append_rotated(cache.handle, 0, [a for a, _ in slots], q, k, v, out)
        plain.append(0, [b for _, b in slots], k.contiguous(), v.contiguous())
        want, size = rotate64(k, [n + step for n in lens], rot, interleaved)
        for i, x in enumerate(history):
            x.append((want[i:i + 1], size[i:i + 1]))
    for (a, b), x in zip(slots, history):
        check_codes(cache, plain, a, b, torch.cat([w for w, _ in x]), torch.cat([s for _, s in x]), k_scale, S, W)
    assert cache.status() == 0


def test_rotated_rows_are_attended(rl, hz, cuda_device):
    """Decode after rotated appends: products of rotated heads depend on the distance alone, so a history shifted by
    any number of tokens gives the same attention up to rounding."""
    dev, Hkv, Hq, D = cuda_device, 2, 8, 128
    n, shift = 200, 3000
    cache = hz.PagedCache(1, Hkv, Hq, D, 2, 200, 4000, [1, 1], 4, 60, device=dev)
    table = make_table(rl, D, 4000, dev)
    rl.rlkv_paged_set_rotary(cache.handle, table, 4000, D)
    q, k, v = apart(n, Hq, Hkv, D, 3, dev)
    near = cache.open_seq()
    qr = torch.empty_like(q)
    rl.rlkv_paged_prefill_rotated(cache.handle, 0, near, q, k, v, n, qr)
    got = cache.decode(0, [near], qr[-1:].contiguous())
    # the same at positions shift .. shift + n - 1, attended by a plain softmax in 64 bits
    kr, _ = rotate64(k, np.arange(n) + shift, D, False)
    qs, _ = rotate64(q[-1:], [n - 1 + shift], D, False)
    for j in range(Hq):
        h = j // 4
        s = (kr[:, h] @ qs[0, j]) / np.sqrt(D)
        p = torch.softmax(s, 0)
        want = p @ v[:, h].double().cpu()
        # roundings: q and k to bf16 (2^-8 of each, in the score), P to bf16
        ds = 2 * 2.0 ** -8 * (kr[:, h].abs() @ qs[0, j].abs()) / np.sqrt(D)
        tol = (p * (2 * ds + 2.0 ** -8 + 1e-4)) @ v[:, h].double().cpu().abs() + float((p * ds).sum()) * want.abs()
        assert bool(((got[0, j].double().cpu() - want).abs() <= tol).all())


def test_refusals(rl, hz, cuda_device):
    dev = cuda_device
    cache = hz.PagedCache(1, 2, 8, 128, 2, 8, 200, [1, 0], 4, 60, device=dev)
    s = cache.open_seq()
    q, k, v = apart(3, 8, 2, 128, 1, dev)
    out = torch.empty_like(q)

    def refused(code, call, *args):
        with pytest.raises(rl.RlkvError) as e:
            call(*args)
        assert e.value.code == code
        assert cache.length(0, s) == length

    length = 0
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s], q[:1], k[:1], v[:1], out[:1])   # no rotation set
    table = make_table(rl, 128, 100, dev)
    for rot in (0, 8, 24, 130, 144):
        refused(rl.RLKV_EINVAL, rl.rlkv_paged_set_rotary, cache.handle, table, 100, rot)
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_set_rotary, cache.handle, table, 0, 128)
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_set_rotary, cache.handle, table.data_ptr() + 4, 100, 128)
    rl.rlkv_paged_set_rotary(cache.handle, table, 100, 128)
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s], q[:1], k[:1], v[:1], None)       # q without q_out
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s, s], q[:2], k[:2], v[:2], out[:2])  # twice the same
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [1], q[:1], k[:1], v[:1], out[:1])    # not open
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 1, [s], q[:1], k[:1], v[:1], out[:1])    # no such layer
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s], q[:1].data_ptr() + 2, k[:1], v[:1], out[:1])
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_prefill_rotated, cache.handle, 0, s, q, k, v, 0, out)
    big = [torch.zeros((101, h, 128), dtype=torch.bfloat16, device=dev) for h in (8, 2, 2)]
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_prefill_rotated, cache.handle, 0, s, *big, 101, torch.empty_like(big[0]))  # past the table
    rl.rlkv_paged_prefill_rotated(cache.handle, 0, s, big[0][:100], big[1][:100], big[2][:100], 100, torch.empty_like(big[0]))
    length = 100
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s], q[:1], k[:1], v[:1], out[:1])    # past the table
    with pytest.raises(ValueError):
        rl.rlkv_paged_append_rotated(cache.handle, 0, [s], q[:1].transpose(0, 1), k[:1], v[:1], out[:1])
    with pytest.raises(rl.RlkvError):
        rl.rlkv_rotary_table(inv_freq(128), 10, torch.empty(10, 64, 2))                                          # host memory
    rl.rlkv_paged_set_rotary(cache.handle, None, 0, 128)
    refused(rl.RLKV_EINVAL, rl.rlkv_paged_append_rotated, cache.handle, 0, [s], q[:1], k[:1], v[:1], out[:1])
    # strides that overlap or are not a multiple of eight
    lib = rl.lib
    rl.rlkv_paged_set_rotary(cache.handle, make_table(rl, 128, 200, dev), 200, 128)
    one = np.array([s], np.int32)
    for strides in ((1016, 0, 0), (1028, 0, 0), (0, 248, 0), (0, 0, 252), (-1024, 0, 0)):
        assert lib.rlkv_paged_append_rotated(cache.handle, 0, one.ctypes.data, 1, q.data_ptr(), strides[0], k.data_ptr(), strides[1],
                                             v.data_ptr(), strides[2], out.data_ptr(), 0) == rl.RLKV_EINVAL
    assert cache.length(0, s) == 100
