"""Calls of the operators between a prompt's first token and single-token decoding, as a serving or training
program makes them, with the same operators in plain torch beside them.

Five families, told apart by a case's "op":

  append   queries and keys are normalised per head and rotated by their position, the keys and values go into
           the paged cache, one token for each of n sequences
  rotate   the same normalisation and rotation of packed tokens on their own: of training samples, with the
           gradients behind it, or of the chunks of several sequences on top of what the cache holds
  write    chunks of several sequences go into the paged cache, in 16 or in 8 bits
  read     tokens of several sequences come back out of it
  chunk    attention of a chunk of new tokens of each of n sequences over the paged cache and over the chunk
           itself: drafts to be verified, prompts that come in pieces, both beside single tokens

`run(state)` makes one pass: with `own` false in elementary torch operations in 32 bits, with `own` true
through the library's entry points.
"""
import math
import random

import numpy as np
import torch

own = False

DEV = "cuda"
TILE = 64  # tokens per page
ROOM = {1: 32768}  # tokens an append state takes before its sequences are started again (else 8192)
EPS = 1e-6


# ---- the cases -----------------------------------------------------------------------------------

def listed():
    big = dict(kv_heads=8, q_heads=32, head_dim=128, sink=16, window=112)
    seven = dict(kv_heads=4, q_heads=28, head_dim=128, sink=16, window=112)
    small = dict(kv_heads=2, q_heads=8, head_dim=64, sink=4, window=60)
    return [
        # chat with one user: a single token per step and layer, all of it launch latency
        dict(name="append 1", op="append", seqs=1, full=4, rot=128, interleaved=False, fused=True, fp8=False, **big),
        # continuous batching at 48 requests on the 8-bit cache, heads of the 7B configuration
        dict(name="append 48, 8 bits", op="append", seqs=48, full=2, rot=128, interleaved=False, fused=False, fp8=True, **seven),
        # training on packed samples of the small model, forward and backward
        dict(name="rotate 5 samples", op="rotate", train=True, tokens=1777, docs=5, pad=15, full=1, rot=64, interleaved=True, fused=False,
             **small),
        # one long sample of the large model, q and k slices of one projection: a bandwidth-bound pass in each direction
        dict(name="rotate 8192", op="rotate", train=True, tokens=8192, docs=1, pad=0, full=8, rot=128, interleaved=False, fused=True, **big),
        # 24 requests come back from another machine and go into the 8-bit cache
        dict(name="write 24 requests, 8 bits", op="write", seqs=24, longest=1500, ragged=True, full=4, fused=False, fp8=True, **big),
        # one long request in 16 bits, as slices of one projection
        dict(name="write 1 x 16384", op="write", seqs=1, longest=16384, ragged=False, full=6, fused=True, fp8=False, **big),
        # the requests that make room for others are read back, 8 bits
        dict(name="read 24 requests, 8 bits", op="read", seqs=24, longest=1500, ragged=True, skip=0.0, full=4, fp8=True, **big),
        # the second half of a shared document, for a prompt on top of it
        dict(name="read 1 x 16384", op="read", seqs=1, longest=16384, ragged=False, skip=0.5, full=6, fp8=False, **big),
        # five drafted tokens of one long request are verified: few rows, the cache's length has to be split
        dict(name="verify 5 of 8192", op="chunk", seqs=1, longest=8192, ragged=False, kind="even", chunk=5, full=6, cap=0.0, bias=False,
             fp8=False, **big),
        # four drafted tokens of each of 32 requests on the 8-bit cache, scores lowered by distance
        dict(name="verify 4 of 32 ragged, 8 bits", op="chunk", seqs=32, longest=14338, ragged=True, kind="even", chunk=4, full=6, cap=0.0,
             bias=True, fp8=True, **big),
        # a piece of one prompt beside 47 requests that decode a token each, capped scores, the 7B configuration
        dict(name="512 beside 47", op="chunk", seqs=48, longest=6000, ragged=True, kind="mixed", chunk=512, full=3, cap=50.0, bias=False,
             fp8=False, **seven),
        # a piece of a long prompt, every head full: the matrix products are the time
        dict(name="2048 on 8192", op="chunk", seqs=1, longest=8192, ragged=False, kind="even", chunk=2048, full=8, cap=0.0, bias=False,
             fp8=False, **big),
    ]


MOST_FLOPS, MOST_BYTES = 3.0e11, 5.0e8  # what the largest listed cases cost


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "rotate", "rotate", "write", "read", "chunk", "chunk", "chunk", "chunk"])
    kv_heads, q_heads, head_dim = rng.choice([(8, 32, 128), (4, 28, 128), (2, 8, 64), (2, 2, 128), (4, 16, 64)])
    sink, window = rng.choice([(16, 112), (4, 60), (16, 240), (0, 5)])
    c = dict(op=op, kv_heads=kv_heads, q_heads=q_heads, head_dim=head_dim, full=rng.randint(0, kv_heads), sink=sink, window=window)
    rotation = dict(rot=rng.choice([head_dim, head_dim, head_dim // 2]), interleaved=rng.random() < 0.3)
    fused, fp8 = rng.random() < 0.5, head_dim == 128 and rng.random() < 0.4
    if op == "append":
        c.update(seqs=_log(rng, 1, 96), fused=fused, fp8=fp8, **rotation)
    elif op == "rotate" and rng.random() < 0.6:
        tokens = _log(rng, 1, 8192)
        c.update(train=True, tokens=tokens, docs=min(tokens, _log(rng, 1, 32)), pad=rng.choice([0, 0, 1, 77]), fused=fused, **rotation)
    elif op in ("write", "read"):
        c.update(seqs=_log(rng, 1, 32), longest=_log(rng, 1, 16384), ragged=rng.random() < 0.7, fp8=fp8)
        c.update(dict(fused=fused) if op == "write" else dict(skip=rng.choice([0.0, 0.0, 0.37, 0.9])))
    else:
        kind = rng.choice(["even", "even", "mixed", "ragged"])
        seqs = rng.choice([1, 2, 3]) if kind == "ragged" else _log(rng, 1, 48)
        chunk = {"even": _log(rng, 1, 16), "mixed": _log(rng, 1, 1024), "ragged": _log(rng, 1, 2048)}[kind]
        c.update(seqs=seqs, longest=rng.choice([0, _log(rng, 1, 16384), _log(rng, 1, 16384)]), ragged=rng.random() < 0.6, kind=kind, chunk=chunk)
        if op == "chunk":
            c.update(cap=rng.choice([0.0, 0.0, 30.0, 50.0]), bias=rng.random() < 0.4, fp8=fp8)
        else:
            c.update(train=False, fused=fused, **rotation)
    while work(c)["flops"] > MOST_FLOPS or work(c)["bytes"] > MOST_BYTES:
        c["longest"] //= 2
    return c


def _spread(n, top):
    """n lengths from `top` down to an eighth of it."""
    return np.round(top * (1 - 0.875 * np.arange(n) / max(1, n - 1))).astype(np.int64)


def _lens(c):
    """Tokens of the sequences of a write, read or chunk case (a chunk's: before the call)."""
    n, top = c["seqs"], c["longest"]
    lens = _spread(n, top) if c["ragged"] else np.full(n, top)
    return lens if c["op"] in ("chunk", "rotate") else np.maximum(1, lens)


def _counts(c):
    """New tokens of each sequence of a chunk."""
    n, m = c["seqs"], c["chunk"]
    if c["kind"] == "even":
        return np.full(n, m)
    if c["kind"] == "ragged":
        return np.maximum(1, _spread(n, m))[::-1].copy()
    counts = np.ones(n, np.int64)
    counts[n // 2] = m
    return counts


def _doc_lens(c):
    """Lengths of the samples: cut at places that go by the case alone."""
    rng = random.Random("%d %d" % (c["tokens"], c["docs"]))
    cuts = sorted(rng.sample(range(1, c["tokens"]), c["docs"] - 1)) if c["docs"] > 1 else []
    return np.diff(np.array([0] + cuts + [c["tokens"]]))


def _full_heads(c):
    """Which KV heads are full: spread over the head index."""
    h = np.arange(c["kv_heads"])
    return ((h * 5 + 1) % c["kv_heads"] < c["full"]) if c["kv_heads"] % 5 else h < c["full"]


def _scale8(c, which):
    """Scales of an 8-bit cache, one per KV head."""
    return (0.009 + 0.001 * ((np.arange(c["kv_heads"]) * 3 + which) % 7)).astype(np.float32)


def _slopes(c):
    """Distance slopes 2^(-8 (j + 1) / heads) of the query heads."""
    return (2.0 ** (-8.0 * (np.arange(c["q_heads"]) + 1) / c["q_heads"])).astype(np.float32)


def _start_lens(c):
    """Tokens the sequences of an append case hold before the pass."""
    return 200 + (np.arange(c["seqs"]) * 37) % 300


def _first(c):
    """The first token that a read case wants of each sequence."""
    return (_lens(c) * c["skip"]).astype(np.int64)


def work(c):
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    each = 1 if c.get("fp8") else 2
    cap = c["sink"] + c["window"]
    if c["op"] == "append":  # q in and out, k and v in, K and V rows stored, the angles
        n = c["seqs"]
        return {"bytes": n * (2 * Hq + 2 * Hkv) * D * 2 + n * Hkv * 2 * D * each + n * c["rot"] * 4,
                "flops": n * (Hq + Hkv) * (3 * c["rot"] + 4 * D)}
    if c["op"] == "rotate":
        n = c["tokens"] if c["train"] else int(_counts(c).sum())
        once = n * (Hq + Hkv) * D * 2
        return {"bytes": once * (4 if c["train"] else 2) + n * c["rot"] * 4, "flops": (3 if c["train"] else 1) * n * (Hq + Hkv) * (3 * c["rot"] + 4 * D)}
    if c["op"] in ("write", "read"):
        lens = _lens(c)
        kept = int(lens.sum()) * c["full"] + int(np.minimum(lens, cap).sum()) * (Hkv - c["full"])
        if c["op"] == "write":
            return {"bytes": kept * 2 * D * (2 + each), "flops": kept * 2 * D}
        first = _first(c)
        lo = np.maximum(first, lens - c["window"])
        seen = int((lens - first).sum()) * c["full"]
        seen += int((lens - lo + np.maximum(0, np.minimum(c["sink"], lo) - first)).sum()) * (Hkv - c["full"])
        return {"bytes": seen * 2 * D * each + int((lens - first).sum()) * Hkv * 2 * D * 2, "flops": seen * 2 * D}
    lens, counts = _lens(c), _counts(c)
    rows = int(lens.sum()) * c["full"] + int(np.minimum(lens, cap).sum()) * (Hkv - c["full"])
    pairs = [0, 0]  # visible (query, key) pairs of a compressed and of a full head
    for n, m in zip(lens.tolist(), counts.tolist()):
        pos = n + np.arange(m)
        lo = np.maximum(pos - c["window"] + 1, 0)
        pairs[1] += int((pos + 1).sum())
        pairs[0] += int((pos + 1 - lo + np.minimum(c["sink"], lo)).sum())
    t = int(counts.sum())
    return {"bytes": rows * 2 * D * each + t * (2 * Hq + 2 * Hkv) * D * 2 + t * Hq * 4,
            "flops": 4 * D * (Hq // Hkv) * (pairs[1] * c["full"] + pairs[0] * (Hkv - c["full"]))}


# ---- what a program has in hand before the call ---------------------------------------------------

class State:
    pass


class _Handle:
    """A handle of the library, given back when the state goes."""

    def __init__(self, destroy, h):
        self.destroy, self.h = destroy, h

    def __del__(self):
        self.destroy(self.h)


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _tokens(n, c, g):
    """q, k, v of n tokens: apart, or slices of one projection's output."""
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c.get("fused"):
        x = _randn((n, Hq + 2 * Hkv, D), g)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return _randn((n, Hq, D), g), _randn((n, Hkv, D), g), _randn((n, Hkv, D), g)


def _weights(c, g):
    """The norms' weights, around one."""
    return (1 + 0.2 * torch.randn((2, c["head_dim"]), generator=g, device=DEV)).unbind(0)


def _inv_freq(c):
    return 10000.0 ** (-np.arange(0, c["rot"], 2) / c["rot"])


def _device_table(c, rows):
    """cos and sin of every position, computed in 64 bits: [rows][rot / 2][2]."""
    a = torch.arange(rows, device=DEV, dtype=torch.float64)[:, None] * torch.from_numpy(_inv_freq(c)).to(DEV)
    return torch.stack([a.cos(), a.sin()], -1).float().contiguous()


def _codes(x, scale, heads_dim=-2):
    """E4M3 codes of x (64 or 32 bits), heads along `heads_dim`."""
    shape = [1] * x.dim()
    shape[heads_dim] = -1
    inv = torch.from_numpy(np.float32(1.0) / scale).to(x.device).reshape(shape)
    return (x * inv.to(x.dtype)).clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _append_plan(c):
    """Pages of the sequences of an append case, in the order in which the cache hands them out: at the
    start sequence by sequence, then wherever a token opens a page."""
    lens, n = _start_lens(c), c["seqs"]
    room = ROOM.get(n, 8192)
    first = -(-lens // TILE)
    most = -(-(lens + room) // TILE)
    table = np.zeros((n, int(most.max())), np.int64)
    base = np.concatenate([[0], np.cumsum(first)])
    opened = []
    for i in range(n):
        table[i, :first[i]] = base[i] + np.arange(first[i])
        j = np.arange(first[i], most[i])
        opened.append(np.stack([j * TILE - lens[i], np.full(j.size, i), j], 1))
    ev = np.concatenate(opened)
    ev = ev[np.lexsort((ev[:, 1], ev[:, 0]))]
    table[ev[:, 1], ev[:, 2]] = base[-1] + np.arange(len(ev))
    return lens, room, int(base[-1]) + len(ev), table


def _whole_plan(lens):
    """Pages of sequences written in one go: sequence by sequence."""
    pages = -(-lens // TILE)
    base = np.concatenate([[0], np.cumsum(pages)])
    table = np.zeros((len(lens), int(pages.max())), np.int64)
    for i, p in enumerate(pages):
        table[i, :p] = base[i] + np.arange(p)
    return int(base[-1]), table


def _ring_row(t, c):
    return torch.where(t < c["sink"], t, c["sink"] + (t - c["sink"]) % c["window"])


def _shapes(c, seqs, pages):
    nf, D = int(_full_heads(c).sum()), c["head_dim"]
    rows = -(-(c["sink"] + c["window"]) // TILE) * TILE
    return (nf, pages, 2, TILE, D), (seqs, c["kv_heads"] - nf, 2, rows, D)


def _of(lens):
    """Sequence and position of packed tokens."""
    return (torch.from_numpy(np.repeat(np.arange(len(lens)), lens)).to(DEV),
            torch.from_numpy(np.concatenate([np.arange(x) for x in lens])).to(DEV))


def _cache(s, c, seqs, pages, longest):
    """The paged cache of a case: the library's handle, or its pages and rings as plain tensors."""
    full_shape, ring_shape = _shapes(c, seqs, pages)
    kind = torch.float8_e4m3fn if c["fp8"] else torch.bfloat16
    if not own:
        s.pool, s.ring = (torch.zeros(x, dtype=torch.float32, device=DEV).to(kind) for x in (full_shape, ring_shape))
        s.heads_full = torch.from_numpy(np.flatnonzero(s.full)).to(DEV)
        s.heads_ring = torch.from_numpy(np.flatnonzero(~s.full)).to(DEV)
        return
    rl = s.rl
    shape = (1, c["kv_heads"], c["q_heads"], c["head_dim"], seqs, pages, longest, s.full.astype(np.uint8), c["sink"], c["window"])
    size = (rl.rlkv_paged_size_fp8 if c["fp8"] else rl.rlkv_paged_size)(*shape)
    s.buf = torch.empty(size + 1024, dtype=torch.uint8, device=DEV)
    s.buf = s.buf[-s.buf.data_ptr() % 1024:][:size]
    s.handle = _Handle(rl.rlkv_paged_destroy,
                       rl.rlkv_paged_create_fp8(*shape, _scale8(c, 0), _scale8(c, 1), s.buf, size) if c["fp8"]
                       else rl.rlkv_paged_create(*shape, s.buf, size))
    n_full, n_ring, each = math.prod(full_shape), math.prod(ring_shape), 1 if c["fp8"] else 2
    s.pool = s.buf[:n_full * each].view(kind).view(full_shape)
    s.ring = s.buf[n_full * each:(n_full + n_ring) * each].view(kind).view(ring_shape)


def _fill(s, k, v, lens):
    """Sequences of these lengths, opened in order and filled with the packed rows of k and v."""
    rl, h = s.rl, s.handle.h
    s.slots = np.array([rl.rlkv_paged_seq_open(h) for _ in lens], np.int32)
    at = 0
    for x, n in zip(s.slots, lens):
        if n:
            rl.rlkv_paged_prefill(h, 0, int(x), k[at:at + n], v[at:at + n], int(n))
        at += n


def _refill(s):
    """The sequences of an append case at their start lengths: at first, and when one has no room left."""
    if s.slots is not None:
        for x in s.slots:
            s.rl.rlkv_paged_seq_close(s.handle.h, int(x))
    _fill(s, s.start[0], s.start[1], s.lens)
    s.step = 0


def prepare(case, seed):
    c, s = dict(case), State()
    s.c = c
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    s.full = _full_heads(c)
    if own:
        import paper_2510_08525_b200.binding as rl
        s.rl = rl
    {"append": _prepare_append, "rotate": _prepare_rotate, "write": _prepare_write, "read": _prepare_read, "chunk": _prepare_chunk}[c["op"]](s, c, g)
    return s


def _prepare_append(s, c, g):
    s.lens, s.room, pages, table = _append_plan(c)
    n, longest = len(s.lens), int(s.lens.max()) + s.room
    s.step, s.slots = 0, None
    s.table = _device_table(c, longest)
    s.q, s.k, s.v = _tokens(n, c, g)
    s.start = _randn((2, int(s.lens.sum()), c["kv_heads"], c["head_dim"]), g)  # the rows the cache holds already
    s.q_weight, s.k_weight = _weights(c, g)
    s.q_out = torch.empty(s.q.shape, dtype=torch.bfloat16, device=DEV)
    _cache(s, c, n, pages, longest)
    if own:
        s.rl.rlkv_paged_set_rotary(s.handle.h, s.table, longest, c["rot"], c["interleaved"])
        s.rl.rlkv_paged_set_norms(s.handle.h, s.q_weight, s.k_weight, EPS)
        _refill(s)
        return
    s.pages = torch.from_numpy(table).to(DEV)
    s.pos0, s.seq = torch.from_numpy(s.lens).to(DEV), torch.arange(n, device=DEV)
    seq, pos = _of(s.lens)
    _store(s, s.start[0].float(), s.start[1].float(), seq, pos, (pos < c["sink"]) | (pos >= s.pos0[seq] - c["window"]))


def _positions(c):
    """Positions of the packed tokens of a rotate case (-1: of no sample), and rows of the table."""
    if c["train"]:
        lens = _doc_lens(c)
        pos = np.concatenate([np.arange(x) for x in lens] + [np.full(c["pad"], -1)])
        return pos, int(lens.max())
    lens, counts = _lens(c), _counts(c)
    return np.concatenate([n + np.arange(m) for n, m in zip(lens, counts)]), int((lens + counts).max())


def _prepare_rotate(s, c, g):
    pos, rows = _positions(c)
    n, Hq, Hkv, D = len(pos), c["q_heads"], c["kv_heads"], c["head_dim"]
    s.table = _device_table(c, rows)
    s.pos = torch.from_numpy(pos.astype(np.int32)).to(DEV)
    s.q, s.k, _ = _tokens(n, c, g)
    s.q_weight, s.k_weight = _weights(c, g)
    s.q_out, s.k_out = (torch.zeros(x.shape, dtype=torch.bfloat16, device=DEV) for x in (s.q, s.k))
    if c["train"]:
        s.dq_out, s.dk_out = _randn((n, Hq, D), g), _randn((n, Hkv, D), g)
        if c["fused"]:  # the gradient of the projection's output, in one piece
            d = torch.zeros((n, Hq + 2 * Hkv, D), dtype=torch.bfloat16, device=DEV)
            s.dq, s.dk = d[:, :Hq], d[:, Hq:Hq + Hkv]
        else:
            s.dq, s.dk = (torch.zeros(x.shape, dtype=torch.bfloat16, device=DEV) for x in (s.q, s.k))
        s.dq_weight, s.dk_weight = (torch.empty(D, dtype=torch.float32, device=DEV) for _ in range(2))
    if not own:
        return
    rl = s.rl
    if c["train"]:
        s.handle = _Handle(rl.rlkv_prompt_destroy, rl.rlkv_prompt_create(1, Hkv, Hq, D, n, s.full.astype(np.uint8), c["sink"], c["window"]))
        rl.rlkv_prompt_set_rotary(s.handle.h, s.table, rows, c["rot"], c["interleaved"])
        rl.rlkv_prompt_set_norms(s.handle.h, s.q_weight, s.k_weight, EPS)
        return
    lens, s.counts = _lens(c), _counts(c)
    pages, _ = _whole_plan(np.maximum(1, lens))
    _cache(s, {**c, "fp8": False}, len(lens), pages, rows)
    rl.rlkv_paged_set_rotary(s.handle.h, s.table, rows, c["rot"], c["interleaved"])
    rl.rlkv_paged_set_norms(s.handle.h, s.q_weight, s.k_weight, EPS)
    held = _randn((int(lens.sum()), Hkv, D), g)
    _fill(s, held, held, lens)


def _prepare_write(s, c, g):
    s.lens = _lens(c)
    pages, table = _whole_plan(s.lens)
    _, s.k, s.v = _tokens(int(s.lens.sum()), c, g)
    _cache(s, c, len(s.lens), pages, int(s.lens.max()))
    if not own:
        s.pages = torch.from_numpy(table).to(DEV)
        s.seq, s.pos = _of(s.lens)
        n = torch.from_numpy(s.lens).to(DEV)[s.seq]
        s.keep = (s.pos < c["sink"]) | (s.pos >= n - c["window"])


def _prepare_read(s, c, g):
    s.lens, s.first = _lens(c), _first(c)
    s.counts = s.lens - s.first
    pages, table = _whole_plan(s.lens)
    k, v = (_randn((int(s.lens.sum()), c["kv_heads"], c["head_dim"]), g) for _ in range(2))
    _cache(s, c, len(s.lens), pages, int(s.lens.max()))
    if own:
        _fill(s, k, v, s.lens)
        s.k_out, s.v_out = (torch.empty((int(s.counts.sum()), c["kv_heads"], c["head_dim"]), dtype=torch.bfloat16, device=DEV) for _ in range(2))
        return
    s.pages = torch.from_numpy(table).to(DEV)
    seq, pos = _of(s.lens)
    n = torch.from_numpy(s.lens).to(DEV)
    _store(s, k.float(), v.float(), seq, pos, (pos < c["sink"]) | (pos >= n[seq] - c["window"]))
    s.seq, s.pos = _of(s.counts)
    s.pos = s.pos + torch.from_numpy(s.first).to(DEV)[s.seq]
    s.keep = (s.pos < c["sink"]) | (s.pos >= n[s.seq] - c["window"])
    s.scales = [torch.from_numpy(_scale8(c, w)).to(DEV)[:, None] for w in (0, 1)] if c["fp8"] else None


def _prepare_chunk(s, c, g):
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    s.lens, s.counts = _lens(c), _counts(c)
    t = int(s.counts.sum())
    held_k, held_v = (_randn((int(s.lens.sum()), Hkv, D), g) for _ in range(2))
    s.q, s.k, s.v = _tokens(t, {**c, "fused": True}, g)
    slopes = _slopes(c) if c["bias"] else None
    if own:
        rl = s.rl
        pages, _ = _whole_plan(np.maximum(1, s.lens))
        _cache(s, c, len(s.lens), pages, int((s.lens + s.counts).max()))
        _fill(s, held_k, held_v, s.lens)
        rl.rlkv_paged_set_scores(s.handle.h, c["cap"], slopes)
        s.out = torch.empty((t, Hq, D), dtype=torch.bfloat16, device=DEV)
        s.lse = torch.empty((t, Hq), dtype=torch.float32, device=DEV)
        return
    if c["fp8"]:
        held_k, held_v = _codes(held_k.float(), _scale8(c, 0)), _codes(held_v.float(), _scale8(c, 1))
    s.scales = [torch.from_numpy(_scale8(c, w)).to(DEV)[:, None] for w in (0, 1)] if c["fp8"] else None
    s.held = [x.split(s.lens.tolist()) for x in (held_k, held_v)]
    s.new = [x.split(s.counts.tolist()) for x in (s.q, s.k, s.v)]
    s.head_full = torch.from_numpy(s.full).to(DEV)
    s.slopes = torch.from_numpy(slopes).to(DEV) if c["bias"] else None


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    return {"append": _append, "rotate": _rotate, "write": _write, "read": _read, "chunk": _chunk}[s.c["op"]](s)


def _normed(x, weight):
    """x [tokens][heads][dim] over the root of its mean square, times the weight; and that factor."""
    r = (x.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return x * r * weight, r


def _turn(x, cos, sin, c):
    """x [tokens][heads][dim] with its first `rot` elements rotated pairwise."""
    r, cos, sin = c["rot"], cos[:, None], sin[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _bits(x, c):
    return x.view(torch.uint8) if c["fp8"] else x


def _places(s, seq, pos):
    """Of each head class: the store, its KV heads, and a function from a subset of the tokens to the views of the store's K and V
    rows and the indices of the tokens' rows in them."""
    c = s.c
    page = s.pages[seq, pos // TILE]
    for pool, heads, paged in ((s.pool, s.heads_full, True), (s.ring, s.heads_ring, False)):
        if heads.numel() == 0:
            continue
        mem = _bits(pool, c)
        row = (pos % TILE if paged else _ring_row(pos, c))[:, None]
        h = torch.arange(heads.numel(), device=DEV)[None]
        index = (h, page[:, None]) if paged else (seq[:, None], h)
        if c["fp8"]:  # tiles of 64 rows of K codes and the V codes of the same rows transposed
            t = mem.view(mem.shape[0], mem.shape[1], -1, 2, TILE * c["head_dim"])
            views = t[:, :, :, 0].unflatten(-1, (TILE, c["head_dim"])), t[:, :, :, 1].unflatten(-1, (c["head_dim"], TILE)).transpose(-1, -2)
            index = (*index, row // TILE, row % TILE)
        else:
            views, index = (mem[:, :, 0], mem[:, :, 1]), (*index, row)
        yield heads, paged, views, index


def _store(s, k, v, seq, pos, keep):
    """K and V rows of tokens `pos` of sequences `seq` into the pages and, where `keep`, into the rings."""
    c = s.c
    if c["fp8"]:
        k, v = _codes(k, _scale8(c, 0)), _codes(v, _scale8(c, 1))
    else:
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
    for heads, paged, views, index in _places(s, seq, pos):
        of = slice(None) if paged else keep
        index = tuple(x if x.shape[0] == 1 and seq.shape[0] != 1 else x[of] for x in index)
        for view, x in zip(views, (k, v)):
            view[index] = _bits(x, c)[of][:, heads]


def _append(s):
    c = s.c
    if own:
        if s.step == s.room:
            _refill(s)
        s.step += 1
        s.rl.rlkv_paged_append_rotated(s.handle.h, 0, s.slots, s.q, s.k, s.v, s.q_out)
        return {"q": s.q_out, "pool": s.pool, "ring": s.ring}
    pos = s.pos0 + s.step
    s.step = (s.step + 1) % s.room
    cos, sin = s.table[pos].unbind(-1)
    q = _turn(_normed(s.q.float(), s.q_weight)[0], cos, sin, c).to(torch.bfloat16)
    k = _turn(_normed(s.k.float(), s.k_weight)[0], cos, sin, c)
    _store(s, k, s.v.float(), s.seq, pos, torch.ones_like(pos, dtype=torch.bool))
    return {"q": q, "pool": s.pool, "ring": s.ring}


def _rotate(s):
    c = s.c
    if own:
        rl, h = s.rl, s.handle.h
        if not c["train"]:
            rl.rlkv_paged_rotate_chunks(h, 0, s.slots, s.counts, s.q, s.k, s.q_out, s.k_out)
            return {"q": s.q_out, "k": s.k_out}
        rl.rlkv_prompt_rotate(h, 0, s.q, s.k, s.pos, s.q_out, s.k_out)
        rl.rlkv_prompt_rotate_backward(h, 0, s.q, s.k, s.pos, s.dq_out, s.dk_out, s.dq, s.dk, s.dq_weight, s.dk_weight)
        return {"q": s.q_out, "k": s.k_out, "dq": s.dq, "dk": s.dk, "dq_weight": s.dq_weight, "dk_weight": s.dk_weight}
    mine = (s.pos >= 0)[:, None, None]
    cos, sin = s.table[s.pos.clamp_min(0)].unbind(-1)
    res = {}
    for name, x, weight, d in (("q", s.q, s.q_weight, s.dq_out if c["train"] else None), ("k", s.k, s.k_weight, s.dk_out if c["train"] else None)):
        x = x.float()
        y, r = _normed(x, weight)
        res[name] = _turn(y, cos, sin, c).masked_fill(~mine, 0).to(torch.bfloat16)
        if c["train"]:
            dy = _turn(d.float(), cos, -sin, c).masked_fill(~mine, 0)
            unit = x * r
            res["d%s_weight" % name] = (dy * unit).sum((0, 1))
            dy = dy * weight
            res["d" + name] = (r * (dy - unit * (dy * unit).mean(-1, keepdim=True))).to(torch.bfloat16)
    return res


def _write(s):
    if own:
        rl, h = s.rl, s.handle.h
        slots = np.array([rl.rlkv_paged_seq_open(h) for _ in s.lens], np.int32)
        rl.rlkv_paged_append_chunks(h, 0, slots, s.lens, s.k, s.v)
        for x in slots[::-1]:  # (the last request first: the next pass finds the pages in the same order)
            rl.rlkv_paged_seq_close(h, int(x))
    else:
        _store(s, s.k.float(), s.v.float(), s.seq, s.pos, s.keep)
    return {"pool": s.pool, "ring": s.ring}


def _read(s):
    c = s.c
    if own:
        s.rl.rlkv_paged_read(s.handle.h, 0, s.slots, s.first, s.counts, s.k_out, s.v_out)
        return {"k": s.k_out, "v": s.v_out}
    out = [torch.zeros((s.seq.numel(), c["kv_heads"], c["head_dim"]), dtype=torch.float32, device=DEV) for _ in range(2)]
    for heads, paged, views, index in _places(s, s.seq, s.pos):
        for w, view in enumerate(views):
            x = view[index]
            x = x.view(torch.float8_e4m3fn).float() * s.scales[w][heads] if c["fp8"] else x.float()
            out[w][:, heads] = x if paged else x.masked_fill(~s.keep[:, None, None], 0)
    return {"k": out[0].to(torch.bfloat16), "v": out[1].to(torch.bfloat16)}


def _chunk(s):
    c = s.c
    if own:
        s.rl.rlkv_paged_chunk_attention(s.handle.h, 0, s.slots, s.counts, s.q, s.k, s.v, s.out, s.lse)
        return {"out": s.out, "lse": s.lse}
    Hkv, D = c["kv_heads"], c["head_dim"]
    outs, lses = [], []
    for i, (n, m) in enumerate(zip(s.lens.tolist(), s.counts.tolist())):
        k, v = (x[i].float() * s.scales[w] if c["fp8"] else x[i].float() for w, x in enumerate(s.held))
        k, v = (torch.cat([x, s.new[1 + w][i].float()]).transpose(0, 1)[:, None] for w, x in enumerate((k, v)))
        q = s.new[0][i].float().transpose(0, 1).unflatten(0, (Hkv, -1))                      # [kv head][group][token][dim]
        x = torch.matmul(q, k.transpose(-1, -2)).mul_(1 / math.sqrt(D))
        t = torch.arange(n + m, device=DEV)
        dist = t[n:, None] - t
        if c["cap"]:
            x = x.div_(c["cap"]).tanh_().mul_(c["cap"])
        if c["bias"]:
            x = x.sub_(s.slopes.view(Hkv, -1, 1, 1) * dist)
        seen = (dist >= 0) & (s.head_full.view(-1, 1, 1, 1) | (t < c["sink"]) | (dist < c["window"]))
        x = x.masked_fill_(~seen, -math.inf)
        top = x.amax(-1, keepdim=True)
        p = x.sub_(top).exp_()
        total = p.sum(-1, keepdim=True)
        outs.append((torch.matmul(p, v) / total).flatten(0, 1).transpose(0, 1).to(torch.bfloat16))
        lses.append((top + total.log()).squeeze(-1).flatten(0, 1).T)
    return {"out": torch.cat(outs), "lse": torch.cat(lses)}


# ---- the same in 64 bits, written from the definitions ---------------------------------------------

def exact(case, seed):
    """What run() returns for a new state, in 64 bits."""
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return {"append": _exact_append, "rotate": _exact_rotate, "write": _exact_write, "read": _exact_read, "chunk": _exact_chunk}[c["op"]](c, g)


def _exact_turned(x, weight, pos, c):
    """Normalised and rotated: pairs as complex numbers, times e^(i angle)."""
    r = c["rot"]
    x = x.double()
    x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / c["head_dim"] + EPS) * weight.double()
    angle = (pos.double()[:, None] * torch.from_numpy(_inv_freq(c)).to(DEV))[:, None]
    turn = torch.polar(torch.ones_like(angle), angle)
    first, second = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
    z = torch.complex(first.contiguous(), second.contiguous()) * turn
    head = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], -1)
    return torch.cat([head, x[..., r:]], -1)


def _exact_store(c, lens, rows, pages, table):
    """Pages and rings that hold rows[w][i], the K (w = 0) and V rows of sequence i; an 8-bit cache in units of its scale."""
    full_shape, ring_shape = _shapes(c, len(lens), pages)
    if math.prod(full_shape) > 1 << 29:  # too large to hold in 64 bits
        return None, None
    pool, ring = (torch.zeros(x, dtype=torch.float64, device=DEV) for x in (full_shape, ring_shape))
    full = _full_heads(c)
    for i, n in enumerate(lens.tolist()):
        t = torch.arange(n, device=DEV)
        page = torch.from_numpy(table[i]).to(DEV)[t // TILE]
        last = t[(t < c["sink"]) | (t >= n - c["window"])]
        for w in (0, 1):
            x = rows[w][i].double()
            if c["fp8"]:
                x = x / torch.from_numpy(_scale8(c, w)).to(DEV).double()[:, None]
            for f, h in enumerate(np.flatnonzero(full)):
                pool[f, page, w, t % TILE] = x[:, h]
            for f, h in enumerate(np.flatnonzero(~full)):
                ring[i, f, w, _ring_row(last, c)] = x[last, h]
    if c["fp8"]:  # tiles of K codes and transposed V codes
        pool = torch.stack([pool[:, :, 0].flatten(-2), pool[:, :, 1].transpose(-1, -2).flatten(-2)], 2).view(full_shape)
        tiles = ring.unflatten(3, (-1, TILE))
        ring = torch.stack([tiles[:, :, 0].flatten(-2), tiles[:, :, 1].transpose(-1, -2).flatten(-2)], 3).reshape(ring_shape)
    return pool, ring


def _exact_append(c, g):
    lens, _, pages, table = _append_plan(c)
    q, k, v = _tokens(len(lens), c, g)
    start = _randn((2, int(lens.sum()), c["kv_heads"], c["head_dim"]), g)
    q_weight, k_weight = _weights(c, g)
    pos = torch.from_numpy(lens).to(DEV)
    q, k = _exact_turned(q, q_weight, pos, c), _exact_turned(k, k_weight, pos, c)
    rows = [[torch.cat([old.double(), new[i:i + 1].double()]) for i, old in enumerate(start[w].split(lens.tolist()))] for w, new in ((0, k), (1, v))]
    pool, ring = _exact_store(c, lens + 1, rows, pages, table)
    return {"q": q, "pool": pool, "ring": ring}


def _exact_rotate(c, g):
    pos, _ = _positions(c)
    n, Hq, Hkv, D = len(pos), c["q_heads"], c["kv_heads"], c["head_dim"]
    q, k, _ = _tokens(n, c, g)
    weights = _weights(c, g)
    pos = torch.from_numpy(pos).to(DEV)
    mine = pos >= 0
    douts = [_randn((n, Hq, D), g), _randn((n, Hkv, D), g)] if c["train"] else [None, None]
    res = {}
    for name, x, weight, d in (("q", q, weights[0], douts[0]), ("k", k, weights[1], douts[1])):
        x, weight = x.double().clone().requires_grad_(c["train"]), weight.double().clone().requires_grad_(c["train"])
        y = torch.where(mine[:, None, None], _exact_turned(x, weight, pos, c), 0.0)
        res[name] = y.detach()
        if c["train"]:
            res["d" + name], res["d%s_weight" % name] = torch.autograd.grad(y, (x, weight), d.double())
    return {k: res[k] for k in (("q", "k", "dq", "dk", "dq_weight", "dk_weight") if c["train"] else ("q", "k"))}


def _exact_write(c, g):
    lens = _lens(c)
    pages, table = _whole_plan(lens)
    _, k, v = _tokens(int(lens.sum()), c, g)
    pool, ring = _exact_store(c, lens, [x.split(lens.tolist()) for x in (k, v)], pages, table)
    return {"pool": pool, "ring": ring}


def _exact_read(c, g):
    lens, first, full = _lens(c), _first(c), _full_heads(c)
    out = []
    for w in (0, 1):
        parts = []
        for i, x in enumerate(_randn((int(lens.sum()), c["kv_heads"], c["head_dim"]), g).split(lens.tolist())):
            if c["fp8"]:
                x = _codes(x.float(), _scale8(c, w)).double() * torch.from_numpy(_scale8(c, w)).to(DEV).double()[:, None]
            x = x.double()
            gone = range(c["sink"], max(c["sink"], int(lens[i]) - c["window"]))
            for h in np.flatnonzero(~full):
                x[gone.start:gone.stop, h] = 0
            parts.append(x[int(first[i]):])
        out.append(torch.cat(parts))
    return {"k": out[0], "v": out[1]}


def _exact_chunk(c, g):
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    lens, counts, full, G = _lens(c), _counts(c), _full_heads(c), Hq // Hkv
    held = [_randn((int(lens.sum()), Hkv, D), g) for _ in range(2)]
    if c["fp8"]:
        held = [_codes(x.float(), _scale8(c, w)).float() * torch.from_numpy(_scale8(c, w)).to(DEV)[:, None] for w, x in enumerate(held)]
    t = int(counts.sum())
    q, k, v = _tokens(t, {**c, "fused": True}, g)
    out, lse = (torch.empty(x, dtype=torch.float64, device=DEV) for x in ((t, Hq, D), (t, Hq)))
    a = b = 0
    for n, m in zip(lens.tolist(), counts.tolist()):
        key, query = torch.arange(n + m, device=DEV), n + torch.arange(m, device=DEV)[:, None]
        for h in range(Hkv):
            kk, vv = (torch.cat([held[w][a:a + n, h].double(), x[b:b + m, h].double()]) for w, x in ((0, k), (1, v)))
            hidden = key > query
            if not full[h]:
                hidden = hidden | ((key >= c["sink"]) & (key <= query - c["window"]))
            for j in range(h * G, h * G + G):
                x = q[b:b + m, j].double() @ kk.T / math.sqrt(D)
                if c["cap"]:
                    x = c["cap"] * torch.tanh(x / c["cap"])
                if c["bias"]:
                    x = x - float(_slopes(c)[j]) * (query - key)
                x = torch.where(hidden, -math.inf, x)
                lse[b:b + m, j] = torch.logsumexp(x, -1)
                out[b:b + m, j] = torch.softmax(x, -1) @ vv
        a, b = a + n, b + m
    return {"out": out, "lse": lse}
