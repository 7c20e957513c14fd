"""Refusals of the rotation, score and prompt calls that need no device."""
import numpy as np
import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2510_08525_b200 import build
    build.build()
    import paper_2510_08525_b200.binding as b
    return b


def test_rotation_and_score_calls_refuse_without_a_device(binding):
    b, lib = binding, binding.lib
    f = np.ones(64)
    for call in (lambda: b.rlkv_paged_set_rotary(0, 16, 10, 128), lambda: b.rlkv_paged_set_scores(0, 1.0),
                 lambda: b.rlkv_paged_append_rotated(0, 0, [0], 16, 16, 16, 16, stream=0),
                 lambda: b.rlkv_paged_prefill_rotated(0, 0, 0, 16, 16, 16, 1, 16, stream=0),
                 lambda: b.rlkv_rotary_table(f, 0, 16, stream=0), lambda: b.rlkv_rotary_table(f, 10, 8, stream=0),
                 lambda: b.rlkv_rotary_table(np.ones(65), 10, 16, stream=0), lambda: b.rlkv_rotary_table(f, 10, None, stream=0)):
        with pytest.raises(b.RlkvError) as e:
            call()
        assert e.value.code == b.RLKV_EINVAL
    assert lib.rlkv_rotary_table(f.ctypes.data, 3, 10, 16, 0) == b.RLKV_EINVAL


def test_prompt_calls_refuse_without_a_device(binding):
    b, lib = binding, binding.lib
    m = np.ones(2, np.uint8)
    for call in (lambda: b.rlkv_prompt_destroy(0), lambda: b.rlkv_prompt_kernel_status(0),
                 lambda: b.rlkv_prompt_create(1, 2, 8, 96, 10, m, 4, 60), lambda: b.rlkv_prompt_create(1, 2, 8, 128, 0, m, 4, 60),
                 lambda: b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 0), lambda: b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 60, -1.0)):
        with pytest.raises(b.RlkvError) as e:
            call()
        assert e.value.code == b.RLKV_EINVAL
    with pytest.raises(ValueError):
        b.rlkv_prompt_create(1, 2, 8, 128, 10, [1], 4, 60)
    with pytest.raises(ValueError):
        b.rlkv_prompt_create(1, 2, 8, 128, 10, m, 4, 60, 0.0, np.ones(7))
    assert lib.rlkv_prompt_attention(0, 0, 16, 0, 16, 0, 16, 0, 1, 1, 16, 0, 1, 0, 16, 16, 0) == b.RLKV_EINVAL
    assert lib.rlkv_prompt_attention_backward(0, 0, 16, 0, 16, 0, 16, 0, 1, 1, 16, 0, 1, 0, 16, 16, 16, 16, 16, 16, 0) == b.RLKV_EINVAL


class Rows:
    """Stands for a bf16 tensor in device memory; its address is never read."""

    def __init__(self, shape, stride=None, size=2, device=0, whole=False):
        self.shape, self.size, self.device, self.is_cuda, self.whole = shape, size, device, True, whole
        self.dtype = torch.int32 if whole else torch.bfloat16 if size == 2 else torch.float32
        self.strides = stride or tuple(int(np.prod(shape[i + 1:])) for i in range(len(shape)))

    def stride(self):
        return self.strides

    def data_ptr(self):
        return 4096

    def numel(self):
        return int(np.prod(self.shape))

    def element_size(self):
        return self.size

    def is_floating_point(self):
        return not self.whole

    def is_contiguous(self):
        return True

    def get_device(self):
        return self.device


def test_rows_and_their_strides(binding):
    b = binding
    assert b._rows(None) == (0, 0) and b._rows(64) == (64, 0)
    assert b._rows(Rows((5, 8, 128))) == (4096, 1024)
    assert b._rows(Rows((5, 8, 128), (2048, 128, 1)), 5) == (4096, 2048)
    assert b._rows(Rows((1, 8, 128), (0, 128, 1))) == (4096, 0)
    for bad, least in ((Rows((5, 8, 128), (0, 128, 1)), 1),               # expanded: 0 would stand for contiguous tokens
                       (Rows((5, 8, 128), (1024, 0, 1)), 1), (Rows((5, 8, 128), (1024, 1, 8)), 1), (Rows((5, 1024)), 1),
                       (Rows((5, 8, 128), size=4), 1), (Rows((4, 8, 128)), 5), (np.zeros((5, 8, 128), np.float16), 1)):
        with pytest.raises(ValueError):
            b._rows(bad, least)
    assert b._room(None, 9) == 0 and b._room(64, 9) == 64 and b._room(Rows((3, 3)), 9) == 4096
    for bad in (Rows((2, 4)), Rows((3, 3), size=4), np.zeros(9, np.float16)):
        with pytest.raises(b.RlkvError) as e:
            b._room(bad, 9)
        assert e.value.code == b.RLKV_EINVAL


def test_calls_refuse_tensors_too_small_for_them(binding):
    b = binding
    q, k, starts = Rows((4, 8, 128)), Rows((4, 2, 128)), Rows((2,), size=4, whole=True)
    for call in (lambda: b.rlkv_paged_append_rotated(0, 0, [0, 1, 2, 3, 4], q, k, k, q, stream=0),
                 lambda: b.rlkv_paged_prefill_rotated(0, 0, 0, q, k, k, 5, q, stream=0),
                 lambda: b.rlkv_rotary_table(np.ones(64), 5, Rows((4, 64, 2), size=4), stream=0),
                 lambda: b.rlkv_paged_set_rotary(0, Rows((4, 64, 2), size=4), 5, 128),
                 lambda: b.rlkv_paged_set_rotary(0, Rows((4, 64, 2)), 4, 128),
                 lambda: b.rlkv_prompt_attention(0, 0, q, k, k, Rows((2,), size=4), None, None, q, None, 0),
                 lambda: b.rlkv_prompt_attention(0, 0, q, k, Rows((3, 2, 128)), starts, None, None, q, None, 0)):
        with pytest.raises(ValueError):
            call()


def test_addresses_of_host_arrays(binding):
    a = np.arange(5, dtype=np.int32)
    assert binding._host(a) == a.ctypes.data
    a.flags.writeable = False
    assert binding._host(a) == a.ctypes.data and isinstance(binding._host(a[:0]), int)


def test_the_stream_is_that_of_the_tensors_gpu(binding, monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    assert binding._stream(None) == 100 and binding._stream(None, Rows((1, 1, 64), device=3)) == 103
    assert binding._stream(None, 4096) == 100 and binding._stream(7, Rows((1, 1, 64), device=3)) == 7


def without_the_library(b, calls, error):
    """Every call raises `error` before the library sees it."""
    class Library:
        def __getattr__(self, name):
            def called(*args):
                raise AssertionError(f"{name} was called")
            return called

    lib, b.lib = b.lib, Library()
    try:
        for call in calls:
            with pytest.raises(error) as e:
                call()
            assert error is not b.RlkvError or e.value.code == b.RLKV_EINVAL
    finally:
        b.lib = lib


def of_type(shape, dtype):
    x = Rows(shape, size=dtype.itemsize)
    x.dtype = dtype
    return x


@pytest.mark.parametrize("dtype", [torch.float16, torch.int16, torch.uint16])
def test_other_types_of_the_same_size_are_refused(binding, dtype):
    """16-bit tensors that are not bf16, 32-bit ones that are not fp32: their bits would be taken for numbers of those types."""
    b = binding
    q, k, starts = Rows((4, 8, 128)), Rows((4, 2, 128)), Rows((2,), size=4, whole=True)
    lse, other_lse = of_type((4, 8), torch.float32), of_type((4, 8), torch.int32)
    like = lambda x: of_type(x.shape, dtype)  # noqa: E731
    grads = dict(out=q, lse=lse, dout=q, dq=q, dk=k, dv=k)
    calls = [lambda: b.rlkv_paged_append_rotated(16, 0, [0, 1, 2, 3], q, k, k, like(q), stream=0),
             lambda: b.rlkv_paged_prefill_rotated(16, 0, 0, q, k, k, 4, like(q), None, stream=0),
             lambda: b.rlkv_paged_prefill_rotated(16, 0, 0, q, k, k, 4, q, like(k), stream=0),
             lambda: b.rlkv_prompt_attention(16, 0, q, k, k, starts, None, None, like(q), lse, 0),
             lambda: b.rlkv_prompt_attention(16, 0, q, k, k, starts, None, None, q, other_lse, 0)]
    for name, x in grads.items():
        given = {**grads, name: other_lse if name == "lse" else like(x)}
        calls.append(lambda given=given: b.rlkv_prompt_attention_backward(16, 0, q, k, k, starts, None, None, *given.values(), stream=0))

    without_the_library(b, calls, b.RlkvError)


def test_slopes_of_another_count_are_refused(binding):
    """The library reads layers * q_heads slopes, whatever the array holds."""
    b = binding
    cache = b._handle(16, 3, 2, 8, 128)
    without_the_library(b, [lambda n=n: b.rlkv_paged_set_scores(cache, 0.0, np.full(n, 0.5, np.float32)) for n in (0, 1, 8, 23, 25)] +
                        [lambda: b.rlkv_paged_set_scores(cache, 0.0, 0.5)], ValueError)


def test_a_created_handle_knows_its_shape(binding, monkeypatch):
    b = binding

    class Library:
        def __getattr__(self, name):
            def create(out, *args):
                out._obj.value = 4096
                return 0
            return create

    monkeypatch.setattr(b, "lib", Library())
    shape, rest = (2, 4, 28, 128), (2, 8, 100, [1] * 8, 4, 60)
    for h in (b.rlkv_paged_create(*shape, *rest), b.rlkv_paged_create_fp8(*shape, *rest, [1.0] * 8, [1.0] * 8)):
        assert h == 4096 and isinstance(h, int) and (h.layers, h.kv_heads, h.q_heads, h.head_dim) == shape


def test_rows_of_other_heads_than_the_handles_are_refused(binding):
    """The library reads and writes rows of the handle's heads.  One token's rows, and slices of a projection that are wide enough
    apart for it, would pass the checks of their strides."""
    b, starts = binding, Rows((2,), size=4, whole=True)
    h = b._handle(16, 1, 2, 8, 128)
    wide = lambda n, heads, d=128: Rows((n, heads, d), (12 * 128, d, 1))  # noqa: E731
    calls = []
    for n in (1, 4):
        q, kv, lse = wide(n, 8), wide(n, 2), of_type((n, 8), torch.float32)
        for bad_q, bad_k, bad_v in ((wide(n, 4), kv, kv), (wide(n, 9), kv, kv), (wide(n, 8, 64), kv, kv), (q, wide(n, 1), kv),
                                    (q, kv, wide(n, 1)), (q, wide(n, 2, 64), wide(n, 2, 64)), (q, wide(n, 1), wide(n, 1))):
            out, args = Rows(bad_q.shape), (bad_q, bad_k, bad_v)
            calls += [lambda n=n, args=args, out=out: b.rlkv_paged_append_rotated(h, 0, range(n), *args, out, stream=0),
                      lambda n=n, args=args, out=out: b.rlkv_paged_prefill_rotated(h, 0, 0, *args, n, out, None, stream=0),
                      lambda args=args, out=out, lse=lse: b.rlkv_prompt_attention(h, 0, *args, starts, None, None, out, lse, stream=0),
                      lambda args=args, out=out, lse=lse: b.rlkv_prompt_attention_backward(
                          h, 0, *args, starts, None, None, out, lse, out, out, Rows(args[1].shape), Rows(args[2].shape), stream=0)]
    without_the_library(b, calls, ValueError)


def test_a_created_prompt_handle_knows_its_shape(binding, monkeypatch):
    b, asked = binding, []

    class Library:
        def rlkv_prompt_create(self, out, *args):
            out._obj.value = 4096
            asked.append(args[:4])
            return 0

    monkeypatch.setattr(b, "lib", Library())
    h = b.rlkv_prompt_create(2, 4, 28, 128, 100, [1] * 8, 4, 60)
    assert h == 4096 and (h.layers, h.kv_heads, h.q_heads, h.head_dim) == (2, 4, 28, 128) == asked[0]


def test_tables_of_other_types_are_refused(binding):
    """A 16-bit table has half the bytes that its count of elements says; integers are not angles;
    an empty one holds none."""
    b, calls = binding, []
    tables = [of_type((10, 64, 2), t) for t in (torch.bfloat16, torch.float16, torch.int32, torch.float64)] + [Rows((0, 64, 2), size=4)]
    for table in tables:
        calls += [lambda table=table: b.rlkv_rotary_table(np.ones(64), 10, table, stream=0),
                  lambda table=table: b.rlkv_paged_set_rotary(16, table, 10, 128)]
    without_the_library(b, calls, ValueError)


def test_tensors_of_another_gpu_are_refused(binding, monkeypatch):
    """Every tensor of a call has to be on the GPU of its handle; where the handle is an address alone, on one GPU."""
    b, away = binding, 1
    monkeypatch.setattr(b, "_ptr", lambda x: 0 if x is None else x.data_ptr())
    on_gpu = b._handle(16, 1, 2, 8, 128)
    on_gpu.device = 0
    q, k, starts, lse = Rows((4, 8, 128)), Rows((4, 2, 128)), Rows((2,), size=4, whole=True), of_type((4, 8), torch.float32)
    prefix = Rows((1,), size=4, whole=True)

    def elsewhere(x):
        y = Rows(x.shape, size=x.size, device=away, whole=x.whole)
        y.dtype = x.dtype
        return y

    kinds = [((q, k, k, q), lambda h, a: b.rlkv_paged_append_rotated(h, 0, [0, 1, 2, 3], *a, stream=0)),
             ((q, k, k, q, k), lambda h, a: b.rlkv_paged_prefill_rotated(h, 0, 0, *a[:3], 4, *a[3:], stream=0)),
             ((q, k, k, starts, starts, prefix, q, lse), lambda h, a: b.rlkv_prompt_attention(h, 0, *a, stream=0)),
             ((q, k, k, starts, starts, prefix, q, lse, q, q, k, k), lambda h, a: b.rlkv_prompt_attention_backward(h, 0, *a, stream=0))]
    calls = []
    for args, call in kinds:
        for i in range(len(args)):
            given = tuple(elsewhere(x) if i == j else x for j, x in enumerate(args))
            calls += [lambda call=call, given=given, h=h: call(h, given) for h in (on_gpu, 16)]
        calls.append(lambda call=call, given=tuple(map(elsewhere, args)): call(on_gpu, given))
    without_the_library(b, calls, ValueError)


def test_calls_on_one_handle_share_one_stream(binding, monkeypatch):
    """Without a stream every call goes to the current stream of the handle's GPU, whatever device is current and whatever
    kind of call it is: an append and the decode behind it are in order."""
    b, seen = binding, {}

    class Library:
        def __getattr__(self, name):
            def called(*args):
                if "create" in name:
                    args[0]._obj.value = 4096
                else:
                    seen.setdefault(name, set()).add(args[-1])
                return 0
            return called

    current = [3]
    monkeypatch.setattr(b, "lib", Library())
    monkeypatch.setattr(torch.cuda, "is_available", lambda: True)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: current[0])
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 100 + device, raising=False)
    mask, sizes = [1, 0], (1, 2, 8, 128)
    locked = [b.rlkv_cache_create(*sizes, 1, 100, mask, 4, 60), b.rlkv_cache_create_fp8(*sizes, 1, 100, mask, 4, 60, [1, 1], [1, 1])]
    paged = [b.rlkv_paged_create(*sizes, 2, 8, 100, mask, 4, 60), b.rlkv_paged_create_fp8(*sizes, 2, 8, 100, mask, 4, 60, [1, 1], [1, 1])]
    prompt = b.rlkv_prompt_create(*sizes, 64, mask, 4, 60)
    current[0] = 0
    rows = lambda *shape: Rows(shape, device=3)  # noqa: E731
    q, k, out = rows(1, 8, 128), rows(1, 2, 128), rows(1, 8, 128)
    starts, lse = Rows((2,), size=4, device=3, whole=True), Rows((1, 8), size=4, device=3)
    for h in locked:
        for name in ("rlkv_append", "rlkv_append_overlapped"):
            getattr(b, name)(h, 0, k, k)
        for name in ("rlkv_decode_attention", "rlkv_decode_attention_overlapped", "rlkv_decode_attention_static_scratch"):
            getattr(b, name)(h, 0, q, out)
        b.rlkv_prefill(h, 0, k, k, 1)
        b.rlkv_layer_step_overlapped(h, 0, k, k, q, out)
        b.rlkv_decode_mixed_attention(h, 0, q, lse, out)
        b.rlkv_step(h, k, k, q, out)
        b.rlkv_step_host(h, 16, 16, 16, 16)
        b.rlkv_cache_reset(h)
    for h in paged:
        for k_, q_, out_ in ((k, q, out), (16, 32, 64)):         # tensors, and addresses alone
            b.rlkv_paged_append(h, 0, [0], k_, k_)
            b.rlkv_paged_prefill(h, 0, 0, k_, k_, 1)
            b.rlkv_paged_append_rotated(h, 0, [0], q_, k_, k_, out_)
            b.rlkv_paged_prefill_rotated(h, 0, 0, q_, k_, k_, 1, out_)
            b.rlkv_paged_decode_attention(h, 0, [0], q_, out_)
            b.rlkv_paged_step(h, [0], k_, k_, q_, out_)
    b.rlkv_prompt_attention(prompt, 0, q, k, k, starts, None, None, out, lse)
    b.rlkv_prompt_attention_backward(prompt, 0, q, k, k, starts, None, None, out, lse, out, out, k, k)
    b.rlkv_rotary_table(np.ones(64), 1, Rows((1, 64, 2), size=4, device=3))
    assert len(seen) == 20 and all(streams == {103} for streams in seen.values()), seen
    b.rlkv_paged_append(16, 0, [0], k, k)                          # an address alone: the tensors' GPU
    b.rlkv_paged_decode_attention(16, 0, [0], 16, 16)              # nothing but addresses: the current device
    b.rlkv_paged_append(paged[0], 0, [0], k, k, 7)
    assert seen["rlkv_paged_append"] == {103, 7} and seen["rlkv_paged_decode_attention"] == {103, 100}


def test_a_prompt_of_more_queries_than_keys_is_refused(binding):
    """The call turns as many queries as there are keys; the rest of the returned queries would be whatever the memory held."""
    import paper_2510_08525_b200.harness as hz

    class Tensor(Rows):
        def dim(self):
            return len(self.shape)

    cache = hz.PagedCache.__new__(hz.PagedCache)
    cache.handle, cache.q_heads, cache.kv_heads, cache.head_dim, cache.device = None, 8, 2, 128, torch.device("cuda:0")
    q, k = (lambda n: Tensor((n, 8, 128))), (lambda n: Tensor((n, 2, 128)))
    for args in ((q(5), k(4), k(4)), (q(3), k(4), k(4)), (q(5), k(4), k(5))):
        with pytest.raises(ValueError, match="same tokens"):
            cache.prefill_rotated(0, 0, *args)


def test_a_handle_keeps_its_table_of_angles(binding, monkeypatch):
    """The rotated calls read the table: its memory is not given back while a handle has it."""
    import gc
    import weakref
    b = binding

    class Library:
        def rlkv_paged_set_rotary(self, cache, table, positions, *args):
            return 0 if positions >= 0 else b.RLKV_EINVAL

        def rlkv_strerror(self, rc):
            return b"refused"

    monkeypatch.setattr(b, "lib", Library())
    monkeypatch.setattr(b, "_ptr", lambda x: 0 if x is None else x.data_ptr())
    h, table = b._handle(16, 1, 2, 8, 128), Rows((10, 64, 2), size=4)
    alive = weakref.ref(table)
    b.rlkv_paged_set_rotary(h, table, 10, 128)
    del table
    gc.collect()
    assert alive() is not None
    with pytest.raises(b.RlkvError):
        b.rlkv_paged_set_rotary(h, None, -1, 128)                  # refused: the one before stays set
    gc.collect()
    assert alive() is not None
    b.rlkv_paged_set_rotary(h, None, 0, 128)
    gc.collect()
    assert alive() is None
