"""Prompt attention (rlkv_prompt_*), forward and backward, against the definition in 64 bits.

Tolerances, from the roundings of the arithmetic (half a step of bf16 is 2^-8 of the value):
  forward   P goes into the second product as bf16: 2^-8 sum p |v|; scores and sums in fp32, the exponent off by at
            most 2e-4 for these inputs: 2e-4 sum p |v|; the result is rounded once: 2^-8 |out|.
  lse       fp32: 1e-4 + 1e-6 |lse|.
  backward  P and ds go into their products as bf16; D_i comes from the bf16 result, off by 2^-8 sum |do o|; p off by 5e-4 of
            itself; do.v in fp32, off by 1e-5 sum |do v|; results rounded once.  Each bound is summed with the
            magnitudes it multiplies."""
import numpy as np
import pytest
import torch

from test_gpu_parity import rand_bf16

pytestmark = pytest.mark.gpu
E = 2.0 ** -8


@pytest.fixture(scope="module")
def rl(cuda_device):
    import paper_2510_08525_b200.binding as binding
    return binding


class Prompt:
    def __init__(self, rl, *shape, **kw):
        self.rl, self.h = rl, rl.rlkv_prompt_create(*shape, **kw)

    def __del__(self):
        self.rl.rlkv_prompt_destroy(self.h)


def reference(c, q, k, v, lq, lk, dout):
    """Results in 64 bits and the bounds of their errors, as dicts."""
    dev = q.device
    q, k, v, dout = (x.double() for x in (q, k, v, dout))
    Hq, D, Hkv = q.shape[1], q.shape[2], k.shape[1]
    G, scale = Hq // Hkv, D ** -0.5
    zero = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=dev)  # noqa: E731
    r = dict(out=zero(q), lse=torch.zeros(q.shape[:2], dtype=torch.float64, device=dev), dq=zero(q), dk=zero(k), dv=zero(v))
    tol = {n: zero(x) for n, x in r.items()}
    q0 = k0 = 0
    for d, (a, b) in enumerate(zip(lq, lk)):
        rows, keys = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        i, j = torch.arange(a, device=dev)[:, None] + (b - a), torch.arange(b, device=dev)[None]
        causal = (j < i + 1) | (j < (c["prefix"][d] if c["prefix"] else 0))
        local = causal & ((j < c["sink"]) | (j > i - c["window"]))
        for h in range(Hq):
            kh, vh, qh, do = k[keys, h // G], v[keys, h // G], q[rows, h], dout[rows, h]
            x = qh @ kh.T * scale
            dx = torch.ones_like(x)
            if c["cap"]:
                t = torch.tanh(x / c["cap"])
                x, dx = c["cap"] * t, 1 - t * t
            if c["slopes"] is not None:
                x = x - float(c["slopes"][h]) * (i - j).abs()
            x = x.masked_fill(~(causal if c["mask"][h // G] else local), -np.inf)
            lse = torch.logsumexp(x, 1) if b else torch.full((a,), -np.inf, dtype=torch.float64, device=dev)
            p = torch.exp(x - torch.where(lse == -np.inf, 0.0, lse)[:, None])
            o = p @ vh
            r["out"][rows, h], r["lse"][rows, h] = o, lse
            tol["out"][rows, h] = (E + 2e-4) * (p @ vh.abs()) + E * o.abs()
            tol["lse"][rows, h] = 1e-4 + 1e-6 * torch.where(lse == -np.inf, 0.0, lse).abs()
            ds = p * (do @ vh.T - (do * o).sum(1, keepdim=True)) * dx
            eds = (E + 5e-4) * ds.abs() + p * (E * (do * o).abs().sum(1, keepdim=True) + 1e-5 * (do.abs() @ vh.abs().T)) + 1e-5 * p * ds.abs()
            r["dv"][keys, h // G] += p.T @ do
            tol["dv"][keys, h // G] += (E + 5e-4) * (p.T @ do.abs())
            r["dq"][rows, h] = ds @ kh * scale
            tol["dq"][rows, h] = eds @ kh.abs() * scale
            r["dk"][keys, h // G] += ds.T @ qh * scale
            tol["dk"][keys, h // G] += eds.T @ qh.abs() * scale
    for n in ("dq", "dk", "dv"):
        tol[n] += E * r[n].abs() + 1e-7
    return r, tol


def starts(lens, dev):
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device=dev)


def call(rl, h, layer, q, k, v, qs, ks, prefix, dout, stream=None, fill=7.0):
    out = torch.full(q.shape, fill, dtype=torch.bfloat16, device=q.device)
    lse = torch.full(q.shape[:2], fill, dtype=torch.float32, device=q.device)
    rl.rlkv_prompt_attention(h, layer, q, k, v, qs, ks, prefix, out, lse, stream)
    dq, dk, dv = (torch.full(x.shape, fill, dtype=torch.bfloat16, device=q.device) for x in (q, k, v))
    rl.rlkv_prompt_attention_backward(h, layer, q, k, v, qs, ks, prefix, out, lse, dout, dq, dk, dv, stream)
    return dict(out=out, lse=lse, dq=dq, dk=dk, dv=dv)


def inputs(tq, tk, Hq, Hkv, D, seed, dev):
    q = rand_bf16((tq, Hq, D), seed).to(dev)
    kv = rand_bf16((tk, 2 * Hkv, D), seed + 1).to(dev)
    return q, kv[:, :Hkv], kv[:, Hkv:], rand_bf16((tq, Hq, D), seed + 2).to(dev)


def check(got, want, tol, nq, nk, fill=7.0):
    for name, g in got.items():
        n = nk if name in ("dk", "dv") else nq
        w, t = want[name][:n], tol[name][:n]
        x = g[:n].double()
        none = w == -np.inf
        assert torch.equal(none, x == -np.inf), name
        err = torch.where(none, 0.0, (x - w).abs())
        assert bool((err <= t).all()), (name, float((err / t).nan_to_num(1e9).max()), (err > t).nonzero()[:4].tolist())
        assert bool((g[n:] == fill).all()), name            # rows behind the last document


CASES = [
    # Hkv, Hq, D, sink, window, mask, query lengths, keys beyond the queries, prefix, cap, slope base, pad
    (1, 1, 64, 4, 60, "1", [1], 0, None, 0.0, 0.0, 0),
    (2, 8, 64, 4, 60, "10", [1, 2, 31, 0, 64, 65], 0, None, 0.0, 0.0, 5),
    (2, 8, 64, 0, 5, "01", [333], 0, None, 0.0, 0.4, 0),
    (2, 8, 64, 4, 60, "10", [127, 128, 129, 255, 256, 257], 0, None, 30.0, 0.0, 1),
    (4, 28, 128, 16, 112, "1001", [300, 1, 77], 0, [40, 0, 500], 0.0, 0.0, 3),
    (2, 2, 128, 16, 112, "10", [700, 513], 0, None, 5.0, 0.1, 0),
    (1, 8, 128, 4, 12, "0", [400, 3], 200, None, 0.0, 0.0, 2),
    (2, 4, 128, 0, 1, "01", [150], -40, None, 0.0, 0.2, 9),
    (2, 4, 64, 20, 130, "01", [200, 5, 190], -7, [30, 3, 9], 20.0, 0.1, 0),
    (1, 2, 128, 300, 100, "0", [1500], 0, None, 0.0, 0.0, 0),
    (2, 4, 64, 130, 260, "01", [1100, 900], 333, [700, 0], 0.0, 0.01, 0),
    (1, 1, 128, 16, 112, "1", [2300], 0, None, 50.0, -0.001, 0),
]


@pytest.mark.parametrize("Hkv,Hq,D,S,W,mask,lq,more,prefix,cap,base,pad", CASES)
def test_prompt_forward_and_backward(rl, cuda_device, Hkv, Hq, D, S, W, mask, lq, more, prefix, cap, base, pad):
    dev, mask = cuda_device, [int(x) for x in mask]
    lk = [max(0, n + more) for n in lq]
    nq, nk = sum(lq), sum(lk)
    slopes = (base * 2.0 ** -np.arange(Hq)).astype(np.float32) if base else None
    c = dict(mask=mask, sink=S, window=W, cap=cap, slopes=slopes, prefix=prefix)
    # a second layer, which is the one that is called
    p = Prompt(rl, 2, Hkv, Hq, D, nq + pad, [1 - x for x in mask] + mask, S, W, cap,
               None if slopes is None else np.concatenate([slopes * 0 + 9, slopes]))
    q, k, v, dout = inputs(nq + pad, nk + pad, Hq, Hkv, D, 11, dev)
    for x in (q, dout):
        x[nq:] = float("nan")                                # what lies behind the documents has no effect
    k[nk:], v[nk:] = float("inf"), float("nan")
    qs, ks = starts(lq, dev), starts(lk, dev) if more else None
    pre = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device=dev)
    got = call(rl, p.h, 1, q, k, v, qs, ks, pre, dout)
    want, tol = reference(c, q[:nq], k[:nk], v[:nk], lq, lk, dout[:nq])
    assert rl.rlkv_prompt_kernel_status(p.h) == 0
    check(got, want, tol, nq, nk)
    again = call(rl, p.h, 1, q, k, v, qs, ks, pre, dout)
    for n in got:
        assert torch.equal(got[n].view(torch.int16 if got[n].element_size() == 2 else torch.int32),
                           again[n].view(torch.int16 if got[n].element_size() == 2 else torch.int32)), n
    # without lse, contiguous tensors, on another stream
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device=dev)
    kc, vc = k.contiguous(), v.contiguous()
    torch.cuda.synchronize()
    rl.rlkv_prompt_attention(p.h, 1, q, kc, vc, qs, ks, pre, out, None, s)
    s.synchronize()
    assert torch.equal(out, got["out"])


@pytest.mark.parametrize("Hkv,Hq,D", [(1, 7, 128), (1, 7, 64), (2, 2, 128), (2, 6, 64)])
@pytest.mark.parametrize("lq,lk", [([300], [100]), ([700], [300]), ([300, 700, 256], [100, 300, 1])])
def test_queries_before_the_first_key(rl, cuda_device, Hkv, Hq, D, lq, lk):
    """Documents of many more queries than keys, odd groups: 128 queries that see no key beside 128 that do, in one CTA.  Their
    rows are zeros whatever their queries hold, in every one of many calls."""
    dev, nq, nk = cuda_device, sum(lq), sum(lk)
    mask = [1, 0][:Hkv]
    for full in (mask, [1 - x for x in mask]):
        c = dict(mask=full, sink=4, window=60, cap=0.0, slopes=None, prefix=None)
        p = Prompt(rl, 1, Hkv, Hq, D, nq, full, 4, 60)
        q, k, v, dout = inputs(nq, nk, Hq, Hkv, D, 43, dev)
        got = call(rl, p.h, 0, q, k, v, starts(lq, dev), starts(lk, dev), None, dout)
        want, tol = reference(c, q, k, v, lq, lk, dout)
        check(got, want, tol, nq, nk)
        unseen = torch.cat([torch.arange(a, device=dev) < a - b for a, b in zip(lq, lk)])
        bufs = [torch.full_like(q, 7.0) for _ in range(20)]
        for out in bufs:
            rl.rlkv_prompt_attention(p.h, 0, q, k, v, starts(lq, dev), starts(lk, dev), None, out, None)
        for out in [got["out"], *bufs]:
            assert bool((out[unseen] == 0).all()) and torch.equal(out, got["out"])
        assert bool((got["dq"][unseen] == 0).all()) and rl.rlkv_prompt_kernel_status(p.h) == 0


def test_documents_do_not_touch_one_another(rl, cuda_device):
    """A document's bits are those it has alone, whatever is packed around it, NaN included."""
    dev, Hkv, Hq, D = cuda_device, 2, 8, 128
    lens = [130, 70, 300]
    p = Prompt(rl, 1, Hkv, Hq, D, 600, [1, 0], 16, 48, 30.0, 0.1 * np.ones(Hq, np.float32))
    q, k, v, dout = inputs(500, 500, Hq, Hkv, D, 5, dev)
    bad = [x.clone() for x in (q, k, v, dout)]
    for x in bad:
        x[:130], x[200:] = float("nan"), float("inf")
    packed = call(rl, p.h, 0, *bad[:3], starts(lens, dev), None, None, bad[3])
    alone = call(rl, p.h, 0, *(x[130:200].contiguous() for x in (q, k, v)), starts([70], dev), None, None, dout[130:200].contiguous())
    for n in packed:
        assert torch.equal(packed[n][130:200], alone[n]), n
        assert bool(torch.isfinite(alone[n]).all())
    assert rl.rlkv_prompt_kernel_status(p.h) == 0


@pytest.mark.parametrize("n_docs,Hkv,Hq,D", [(31, 2, 4, 64), (64, 1, 7, 64), (65, 2, 4, 128), (700, 1, 2, 64)])
def test_many_documents(rl, cuda_device, n_docs, Hkv, Hq, D):
    """Short and empty documents, more than a warp's lanes and more than a round of the search."""
    dev = cuda_device
    lq = [(i * 37) % 13 if i % 50 else 150 for i in range(n_docs)]
    lk = [n + 3 * (i % 3) for i, n in enumerate(lq)]
    c = dict(mask=[1, 0][:Hkv], sink=2, window=5, cap=0.0, slopes=None, prefix=None)
    nq, nk = sum(lq), sum(lk)
    p = Prompt(rl, 1, Hkv, Hq, D, nq, c["mask"], 2, 5)
    q, k, v, dout = inputs(nq, nk, Hq, Hkv, D, 17, dev)
    got = call(rl, p.h, 0, q, k, v, starts(lq, dev), starts(lk, dev), None, dout)
    want, tol = reference(c, q, k, v, lq, lk, dout)
    check(got, want, tol, nq, nk)
    assert rl.rlkv_prompt_kernel_status(p.h) == 0


def test_long_document_and_window(rl, cuda_device):
    """Many key tiles: the ring of K and V tiles goes round, sums over query heads go through one CTA's ring too."""
    dev, Hkv, Hq, D, n = cuda_device, 2, 4, 128, 5000
    c = dict(mask=[1, 0], sink=200, window=1000, cap=0.0, slopes=None, prefix=None)
    p = Prompt(rl, 1, Hkv, Hq, D, n, c["mask"], 200, 1000)
    q, k, v, dout = inputs(n, n, Hq, Hkv, D, 19, dev)
    got = call(rl, p.h, 0, q, k, v, starts([n], dev), None, None, dout)
    want, tol = reference(c, q, k, v, [n], [n], dout)
    check(got, want, tol, n, n)


def test_large_scores(rl, cuda_device):
    """One key takes nearly all of a row's weight, later keys raise the running maximum again and again."""
    dev, Hkv, Hq, D, n = cuda_device, 1, 2, 64, 700
    p = Prompt(rl, 1, Hkv, Hq, D, n, [1], 4, 60)
    q, k, v, dout = inputs(n, n, Hq, Hkv, D, 23, dev)
    k = (k.float() * torch.linspace(0.1, 12, n, device=dev)[:, None, None]).to(torch.bfloat16)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=dev)
    rl.rlkv_prompt_attention(p.h, 0, q, k, v, starts([n], dev), None, None, out, lse)
    c = dict(mask=[1], sink=4, window=60, cap=0.0, slopes=None, prefix=None)
    want, tol = reference(c, q, k, v, [n], [n], dout)
    # scores up to about 400 / 8: fp32 products are off by up to 64 * 2^-24 of the sum of magnitudes, 2e-4 in the exponent at most
    assert bool(((out.double() - want["out"]).abs() <= tol["out"] + 4e-4 * want["out"].abs() + 1e-3 * tol["out"]).all())
    assert bool(((lse.double() - want["lse"]).abs() <= 1e-3).all())


@pytest.mark.parametrize("D,cap,more", [(64, 0.0, 0), (128, 30.0, 0), (64, 0.0, 127), (128, 0.0, 255), (128, 30.0, 127)])
def test_steep_slopes(rl, cuda_device, D, cap, more):
    """Slopes up to the largest: the scores of the keys next to the query keep their digits, whatever the far ones come to.
    (With 127 keys before the first query its own key is the last of a tile that lies wholly behind the queries.)"""
    dev, Hkv, Hq, n = cuda_device, 2, 8, 700
    slopes = np.float32([1e6, 1e3, 37, 3, 1e6, 1e4, 100, 0.7])
    c = dict(mask=[1, 0], sink=4, window=200, cap=cap, slopes=slopes, prefix=None)
    p = Prompt(rl, 1, Hkv, Hq, D, n, c["mask"], 4, 200, cap, slopes)
    q, k, v, dout = inputs(n, n + more, Hq, Hkv, D, 29, dev)
    got = call(rl, p.h, 0, q, k, v, starts([n], dev), starts([n + more], dev), None, dout)
    want, tol = reference(c, q, k, v, [n], [n + more], dout)
    check(got, want, tol, n, n + more)


@pytest.mark.parametrize("D,S,W,full,cap", [(128, 0, 5, 0, 50.0), (64, 0, 5, 0, 0.0), (128, 2, 3, 0, 0.0), (64, 4, 60, 1, 0.0)])
def test_gradients_of_queries_that_see_few_keys(rl, cuda_device, D, S, W, full, cap):
    """Documents of one tile: the rounding of `out` does not come back in dQ, which is off by little more than its own rounding."""
    dev, Hkv, Hq, lens = cuda_device, 2, 4, [71, 128, 5, 1, 40]
    n = sum(lens)
    p = Prompt(rl, 1, Hkv, Hq, D, n, [full] * 2, S, W, cap)
    q, k, v, dout = inputs(n, n, Hq, Hkv, D, 37, dev)
    got = call(rl, p.h, 0, q, k, v, starts(lens, dev), None, None, dout)
    at = 0
    for a in lens:
        rows, i, j = slice(at, at + a), torch.arange(a, device=dev)[:, None], torch.arange(a, device=dev)[None]
        at += a
        see = (j <= i) & ((j < S) | (j > i - W) | bool(full))
        for h in range(Hq):
            qh, kh, vh, do = (x[rows, y].double() for x, y in ((q, h), (k, h // 2), (v, h // 2), (dout, h)))
            x, dx = qh @ kh.T * D ** -0.5, 1.0
            if cap:
                t = torch.tanh(x / cap)
                x, dx = cap * t, 1 - t * t
            pr = torch.softmax(x.masked_fill(~see, -np.inf), 1)
            ds = pr * (do @ vh.T - (do * (pr @ vh)).sum(1, keepdim=True)) * dx
            want = ds @ kh * D ** -0.5
            # dS is 2^-17 off as two bf16 parts and 5e-4 with its P; dP, an fp32 sum of 128 products, and the sum of P dP that
            # takes its place in D are off by 1e-5 of what they add up, each
            eds = 6e-4 * ds.abs() + 2e-5 * pr * (do.abs() @ vh.abs().T + (pr * (do.abs() @ vh.abs().T)).sum(1, keepdim=True))
            tol = E * want.abs() + eds @ kh.abs() * D ** -0.5 + 1e-7
            err = (got["dq"][rows, h].double() - want).abs()
            assert bool((err <= tol).all()), (a, h, float((err / tol).max()))


def test_last_row_is_the_decode_step(rl, cuda_device):
    """The last query of a prompt sees what the cache retains: prompt attention, paged decode and the mixed call agree."""
    import paper_2510_08525_b200.harness as hz
    dev, Hkv, Hq, D, n = cuda_device, 2, 8, 128, 500
    slopes = (0.05 * 2.0 ** -np.arange(Hq)).astype(np.float32)
    q, k, v, _ = inputs(n, n, Hq, Hkv, D, 8, dev)
    table = torch.empty((n + 4, D // 2, 2), dtype=torch.float32, device=dev)
    rl.rlkv_rotary_table(10000.0 ** (-np.arange(0, D, 2) / D), n + 4, table)
    cache = hz.PagedCache(1, Hkv, Hq, D, 1, 10, n + 4, [1, 0], 16, 112, device=dev)
    cache_set = cache.handle
    rl.rlkv_paged_set_rotary(cache_set, table, n + 4, D)
    rl.rlkv_paged_set_scores(cache_set, 30.0, slopes)
    s = cache.open_seq()
    qr, kr = torch.empty_like(q), torch.empty((n, Hkv, D), dtype=torch.bfloat16, device=dev)
    rl.rlkv_paged_prefill_rotated(cache_set, 0, s, q, k, v, n, qr, kr)
    p = Prompt(rl, 1, Hkv, Hq, D, n, [1, 0], 16, 112, 30.0, slopes)
    out = torch.empty_like(q)
    rl.rlkv_prompt_attention(p.h, 0, qr, kr, v, starts([n], dev), None, None, out, None)
    got = cache.decode(0, [s], qr[-1:].contiguous())
    want, tol = reference(dict(mask=[1, 0], sink=16, window=112, cap=30.0, slopes=slopes, prefix=None), qr[-1:], kr, v, [1], [n], qr[-1:])
    assert bool(((got[0].double() - want["out"][0]).abs() <= tol["out"][0]).all())
    assert bool(((out[-1].double() - want["out"][0]).abs() <= tol["out"][0]).all())
    # one more token: appended with its rotation, attended, and the same as a prompt piece of one query
    q1, k1, v1, _ = inputs(1, 1, Hq, Hkv, D, 88, dev)
    q1r = torch.empty_like(q1)
    rl.rlkv_paged_append_rotated(cache_set, 0, [s], q1, k1, v1, q1r)
    got = cache.decode(0, [s], q1r)
    rows = cache.export_head(0, s, 0)[0][n:n + 1]               # the appended key as the full head holds it
    k1r = torch.from_numpy(rows.view(np.int16).copy()).view(torch.bfloat16).to(dev)
    both = torch.empty((n + 1, Hkv, D), dtype=torch.bfloat16, device=dev)
    x = torch.empty_like(k1)                                    # rotate the key of the other head by a prompt of its own
    cache2 = hz.PagedCache(1, Hkv, Hq, D, 1, 10, n + 4, [1, 1], 16, 112, device=dev)
    rl.rlkv_paged_set_rotary(cache2.handle, table, n + 4, D)
    s2 = cache2.open_seq()
    cache2.prefill(0, s2, kr, v.contiguous())
    rl.rlkv_paged_append_rotated(cache2.handle, 0, [s2], None, k1, v1, None)
    for h in range(Hkv):
        rows = cache2.export_head(0, s2, h)[0][n]
        x[0, h] = torch.from_numpy(rows.view(np.int16).copy()).view(torch.bfloat16).to(dev)
    assert torch.equal(x[0, 0], k1r[0])
    both[:n], both[n:] = kr, x
    piece = torch.empty_like(q1)
    rl.rlkv_prompt_attention(p.h, 0, q1r, both, torch.cat([v, v1]), starts([1], dev), starts([n + 1], dev), None, piece, None)
    want, tol = reference(dict(mask=[1, 0], sink=16, window=112, cap=30.0, slopes=slopes, prefix=None), q1r, both, torch.cat([v, v1]),
                          [1], [n + 1], q1r)
    for y in (got, piece):
        assert bool(((y.double() - want["out"]).abs() <= tol["out"]).all())
    assert cache.status() == 0 and rl.rlkv_prompt_kernel_status(p.h) == 0


def test_gradients_match_differences(rl, cuda_device):
    """d(sum out * dout) along random directions, by central differences of the definition in 64 bits."""
    dev, Hkv, Hq, D, lens = cuda_device, 2, 4, 64, [90, 150]
    slopes = np.array([0.1, 0.02, 0.3, 0.01], np.float32)
    c = dict(mask=[1, 0], sink=3, window=40, cap=4.0, slopes=slopes, prefix=[10, 0])
    p = Prompt(rl, 1, Hkv, Hq, D, 240, c["mask"], 3, 40, 4.0, slopes)
    q, k, v, dout = inputs(240, 240, Hq, Hkv, D, 21, dev)
    got = call(rl, p.h, 0, q, k, v, starts(lens, dev), None, torch.tensor(c["prefix"], dtype=torch.int32, device=dev), dout)
    _, tol = reference(c, q, k, v, lens, lens, dout)
    base = dict(q=q.double(), k=k.double(), v=v.double())
    g = torch.Generator(device=dev)
    g.manual_seed(1)
    for name in ("q", "k", "v"):
        u = torch.randn(base[name].shape, generator=g, device=dev, dtype=torch.float64)
        eps, vals = 1e-4, []
        for sign in (1, -1):
            x = {**base, name: base[name] + sign * eps * u}
            vals.append(float((reference(c, x["q"], x["k"], x["v"], lens, lens, dout)[0]["out"] * dout.double()).sum()))
        slope = (vals[0] - vals[1]) / (2 * eps)
        # (rounded gradients times u: every element may be off by its bound)
        assert abs(float((got["d" + name].double() * u).sum()) - slope) <= float((tol["d" + name] * u.abs()).sum()) + 1e-3


def test_captured_call_reads_starts_and_inputs_anew(rl, cuda_device):
    dev, Hkv, Hq, D, n = cuda_device, 2, 4, 64, 300
    p = Prompt(rl, 1, Hkv, Hq, D, n, [1, 0], 4, 60)
    q, k, v, dout = (x.contiguous() for x in inputs(n, n, Hq, Hkv, D, 31, dev))
    qs = starts([100, 200], dev)
    bufs = {}
    call(rl, p.h, 0, q, k, v, qs, None, None, dout)              # (first use before the capture)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        bufs = call(rl, p.h, 0, q, k, v, qs, None, None, dout, stream=s)
    for lens, seed in (([100, 200], 31), ([7, 293], 41), ([300, 0], 51)):
        for x, y in zip((q, k, v, dout), inputs(n, n, Hq, Hkv, D, seed, dev)):
            x.copy_(y)
        qs.copy_(starts(lens, dev))
        graph.replay()
        torch.cuda.synchronize()
        eager = call(rl, p.h, 0, q, k, v, qs, None, None, dout)
        for name in eager:
            assert torch.equal(eager[name], bufs[name]), (name, lens)


@pytest.mark.parametrize("Hkv,Hq,D,lens", [(2, 8, 64, [300, 5, 70]), (4, 28, 128, [900]), (1, 1, 128, [2000, 1])])
def test_calls_one_after_the_other(rl, cuda_device, Hkv, Hq, D, lens):
    """The backward pass's launches overlap: calls on other inputs right behind one another, without documents between them,
    give the bits that each gives alone."""
    dev, n = cuda_device, sum(lens)
    p = Prompt(rl, 1, Hkv, Hq, D, n, [1] * Hkv, 4, 60)
    sets = [inputs(n, n, Hq, Hkv, D, 71 + 5 * i, dev) for i in range(3)]
    of = [starts(lens, dev), starts(lens[::-1], dev), torch.zeros(2, dtype=torch.int32, device=dev)]
    alone = []
    for x, s in zip(sets, of):
        alone.append(call(rl, p.h, 0, *x[:3], s, None, None, x[3]))
        torch.cuda.synchronize()
    many = [[call(rl, p.h, 0, *x[:3], s, None, None, x[3]) for x, s in zip(sets, of)] for _ in range(8)]
    for got in many:
        for a, b in zip(got, alone):
            for name in a:
                assert torch.equal(a[name], b[name]), name
    assert rl.rlkv_prompt_kernel_status(p.h) == 0


def test_starts_outside_the_tensors_stay_inside(rl, cuda_device):
    """Starts that run past the tensors or backwards name clipped or empty documents: no row outside is touched."""
    dev, Hkv, Hq, D, n = cuda_device, 1, 2, 64, 100
    p = Prompt(rl, 1, Hkv, Hq, D, n, [1], 4, 60)
    q, k, v, dout = inputs(n, n, Hq, Hkv, D, 61, dev)
    want = call(rl, p.h, 0, q, k, v, starts([60, 40], dev), None, None, dout)
    got = call(rl, p.h, 0, q, k, v, torch.tensor([-5, 60, 1 << 30], dtype=torch.int32, device=dev), None, None, dout)
    for name in want:
        assert torch.equal(got[name], want[name]), name
    back = call(rl, p.h, 0, q, k, v, torch.tensor([100, 60, 20], dtype=torch.int32, device=dev), None, None, dout)
    for name in back:
        assert bool((back[name] == 7).all()), name
    assert rl.rlkv_prompt_kernel_status(p.h) == 0


def test_refusals(rl, cuda_device):
    dev = cuda_device
    ok = dict(layers=1, kv_heads=2, q_heads=8, head_dim=128, max_tokens=64, head_is_full=[1, 0], sink=4, window=60, softcap=0.0, slopes=None)
    for bad in (dict(layers=0), dict(kv_heads=3), dict(q_heads=18), dict(head_dim=96), dict(max_tokens=0), dict(max_tokens=1 << 25),
                dict(sink=-1), dict(window=0), dict(softcap=-1.0), dict(softcap=float("nan")), dict(softcap=1e-5), dict(softcap=2e3),
                dict(slopes=np.full(8, np.nan, np.float32)), dict(slopes=np.full(8, 1e7, np.float32))):
        kw = {**ok, **bad}
        if "kv_heads" in bad:
            kw["head_is_full"] = [1, 0, 1]
        if "layers" in bad:
            kw["head_is_full"] = []
        with pytest.raises(rl.RlkvError) as e:
            rl.rlkv_prompt_create(**kw)
        assert e.value.code == rl.RLKV_EINVAL
    p = Prompt(rl, **ok)
    q, k, v, _ = inputs(64, 64, 8, 2, 128, 3, dev)
    qs = starts([64], dev)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=dev)

    def refused(*args):
        with pytest.raises(rl.RlkvError) as e:
            rl.rlkv_prompt_attention(p.h, *args)
        assert e.value.code == rl.RLKV_EINVAL

    refused(1, q, k, v, qs, None, None, out, lse)
    refused(-1, q, k, v, qs, None, None, out, lse)
    refused(0, q, k, v, qs[:1], None, None, out, lse)                                    # no document
    refused(0, q, k, v, qs, None, None, None, lse)
    refused(0, torch.cat([q, q]), k, v, qs, None, None, out, lse)                        # more than max_tokens
    refused(0, q, k[:0], v[:0], qs, None, None, out, lse)
    with pytest.raises(ValueError):
        rl.rlkv_prompt_attention(p.h, 0, q, k, v, qs.long(), None, None, out, lse)
    with pytest.raises(ValueError):
        rl.rlkv_prompt_attention(p.h, 0, q, k, v, qs.cpu(), None, None, out, lse)        # read on the device
    with pytest.raises(ValueError):
        rl.rlkv_prompt_attention(p.h, 0, q.cpu(), k, v, qs, None, None, out, lse)
    with pytest.raises(ValueError):
        rl.rlkv_prompt_attention(p.h, 0, q, k, v, qs, starts([1, 2], dev), None, out, lse)
    with pytest.raises(ValueError):
        rl.rlkv_prompt_attention(p.h, 0, q.transpose(0, 1), k, v, qs, None, None, out, lse)
    ptr = lambda x: x.data_ptr()  # noqa: E731
    f = rl.lib.rlkv_prompt_attention
    good = [p.h, 0, ptr(q), 0, ptr(k), 512, ptr(v), 512, 64, 64, ptr(qs), 0, 1, 0, ptr(out), ptr(lse), 0]
    assert f(*good) == 0
    for at, x in ((0, 0), (2, 0), (2, ptr(q) + 2), (3, 1016), (3, 1028), (5, 248), (7, 1 << 31), (8, 0), (9, 0), (10, 0), (10, ptr(qs) + 1),
                  (12, 0), (12, 65536), (14, ptr(out) + 8), (15, ptr(lse) + 2)):
        assert f(*(x if i == at else y for i, y in enumerate(good))) == rl.RLKV_EINVAL, (at, x)
    b = rl.lib.rlkv_prompt_attention_backward
    d = torch.empty_like(q), torch.empty((64, 2, 128), dtype=torch.bfloat16, device=dev), torch.empty((64, 2, 128), dtype=torch.bfloat16, device=dev)
    good = good[:16] + [ptr(q), *map(ptr, d), 0]
    assert b(*good) == 0
    for at in (15, 16, 17, 18, 19):
        assert b(*(0 if i == at else y for i, y in enumerate(good))) == rl.RLKV_EINVAL, at
    torch.cuda.synchronize()
