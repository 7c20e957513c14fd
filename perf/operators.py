"""Calls of the operators around the decode path, as a serving or training program makes them, with the
same operators in plain torch beside them.

Three families, told apart by a case's "op":

  append / prefill   keys are rotated by their position and appended to the paged cache, the queries are
                     rotated on the way (one token for each of n sequences, or a prompt of one sequence)
  decode             attention of one new token per sequence over the paged cache, with scores capped by
                     a tanh and lowered by the distance between query and key
  prompt / train     attention over whole prompts packed behind one another (documents), forward alone or
                     forward and backward; every KV head is full or sees sink + window tokens only

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
LOG_ROOM = {1: 32768}  # decode appends a state has room for before its slots are recycled (else 8192)


# ---- the cases -----------------------------------------------------------------------------------

def listed():
    return [
        # chat with one user: a single token per step and layer, all of it launch latency
        dict(name="append 1", op="append", seqs=1, kv_heads=8, q_heads=32, head_dim=128, full=4, sink=16, window=112,
             rot=128, interleaved=False, fused=True, fp8=False),
        # continuous batching at 64 requests on the 8-bit cache, heads of the 7B configuration
        dict(name="append 64, 8 bits", op="append", seqs=64, kv_heads=4, q_heads=28, head_dim=128, full=2, sink=16, window=112,
             rot=128, interleaved=False, fused=False, fp8=True),
        # a long prompt goes into the cache: a bandwidth-bound pass over q, k, v
        dict(name="prefill 8192", op="prefill", tokens=8192, kv_heads=8, q_heads=32, head_dim=128, full=6, sink=16,
             window=112, rot=128, interleaved=False, fused=True, fp8=False),
        # one long request alone on the GPU: few rows, the cache's length has to be split
        dict(name="decode 1 x 8192", op="decode", seqs=1, longest=8192, ragged=False, kv_heads=8, q_heads=32, head_dim=128, full=6,
             sink=16, window=112, cap=50.0, bias=False, fp8=False),
        # a ragged batch on the 8-bit cache, scores lowered by distance
        dict(name="decode 16 ragged, 8 bits", op="decode", seqs=16, longest=14338, ragged=True, kv_heads=8, q_heads=32, head_dim=128,
             full=6, sink=16, window=112, cap=0.0, bias=True, fp8=True),
        # the large batch of the 7B configuration, capped and biased scores
        dict(name="decode 32 x 16384", op="decode", seqs=32, longest=16384, ragged=False, kv_heads=4, q_heads=28, head_dim=128, full=4,
             sink=16, window=112, cap=30.0, bias=True, fp8=False),
        # a short question of odd length on the small model
        dict(name="prompt 333", op="prompt", tokens=333, docs=1, pad=3, context=0, prefix=0, kv_heads=2, q_heads=8, head_dim=64,
             full=1, sink=4, window=60, cap=0.0, bias=True),
        # 24 requests packed into one prefill pass, a shared instruction prefix seen from both sides, half of
        # the heads compressed
        dict(name="prompt 24 documents", op="prompt", tokens=8000, docs=24, pad=56, context=0, prefix=40, kv_heads=8, q_heads=32,
             head_dim=128, full=4, sink=16, window=112, cap=50.0, bias=False),
        # one long prompt, every head full: the matrix products are the time
        dict(name="prompt 8192", op="prompt", tokens=8192, docs=1, pad=0, context=0, prefix=0, kv_heads=8, q_heads=32, head_dim=128,
             full=8, sink=16, window=112, cap=0.0, bias=False),
        # training on packed samples of the small model
        dict(name="train 5 documents", op="train", tokens=1777, docs=5, pad=15, context=0, prefix=33, kv_heads=2, q_heads=8, head_dim=64,
             full=1, sink=4, window=60, cap=30.0, bias=True),
        # one sample, half of the heads local (the local branch while the gates are trained)
        dict(name="train 4096", op="train", tokens=4096, docs=1, pad=0, context=0, prefix=0, kv_heads=8, q_heads=32, head_dim=128,
             full=4, sink=16, window=112, cap=0.0, bias=False),
        # one long reasoning trace, every head full
        dict(name="train 8192", op="train", tokens=8192, docs=1, pad=0, context=0, prefix=0, kv_heads=8, q_heads=32, head_dim=128,
             full=8, sink=16, window=112, cap=0.0, bias=False),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "prefill", "decode", "decode", "prompt", "prompt", "train", "train"])
    kv_heads, q_heads, head_dim = rng.choice([(8, 32, 128), (4, 28, 128), (2, 8, 64), (2, 2, 128), (4, 16, 64)])
    sink, window = rng.choice([(16, 112), (4, 60), (16, 240), (0, 5)])
    c = dict(op=op, kv_heads=kv_heads, q_heads=q_heads, head_dim=head_dim, full=rng.randint(0, kv_heads), sink=sink, window=window)
    if op in ("append", "prefill"):
        c.update(rot=rng.choice([head_dim, head_dim, head_dim // 2]), interleaved=rng.random() < 0.3, fused=rng.random() < 0.5,
                 fp8=head_dim == 128 and rng.random() < 0.4)
        if op == "append":
            c["seqs"] = _log(rng, 1, 96)
        else:
            c["tokens"] = _log(rng, 1, 8192)
    elif op == "decode":
        seqs = _log(rng, 1, 32)
        c.update(seqs=seqs, longest=_log(rng, 1, 16384), ragged=rng.random() < 0.6, cap=rng.choice([0.0, 30.0, 50.0]),
                 bias=rng.random() < 0.5, fp8=head_dim == 128 and rng.random() < 0.4)
    else:
        # (samples to train on are not of a token or two: the gradient of scores that cannot differ is nothing)
        tokens = _log(rng, 64, 6000) if op == "train" else _log(rng, 1, 8000)
        c.update(tokens=tokens, docs=min(max(1, tokens // 32) if op == "train" else tokens, _log(rng, 1, 32)), pad=rng.choice([0, 0, 1, 77]),
                 context=rng.choice([0, 0, 0, 200, -3]), prefix=rng.choice([0, 0, 25, 300]), cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                 bias=rng.random() < 0.4)
    return c


def _doc_lens(c):
    """The documents' query and key lengths: cut at places that go by the case alone."""
    rng = random.Random("%d %d" % (c["tokens"], c["docs"]))
    cuts = sorted(rng.sample(range(1, c["tokens"]), c["docs"] - 1)) if c["docs"] > 1 else []
    lq = np.diff(np.array([0] + cuts + [c["tokens"]]))
    return lq, np.maximum(lq + c["context"], 0)


def _seq_lens(c):
    """Sequence lengths of a decode batch: from an eighth of the longest up."""
    n, top = c["seqs"], c["longest"]
    if not c["ragged"]:
        return np.full(n, top)
    return np.maximum(1, np.round(top * (1 - 0.875 * np.arange(n) / max(1, n - 1)))).astype(np.int64)


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


def work(c):
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    if c["op"] in ("append", "prefill"):
        n = c["seqs"] if c["op"] == "append" else c["tokens"]
        stored = n * Hkv
        if c["op"] == "prefill":  # a compressed head keeps sink + window rows of the prompt
            stored = n * c["full"] + min(n, c["sink"] + c["window"]) * (Hkv - c["full"])
        # q in and out, k in (and, for a prompt, its rotated rows out), K and V rows stored, the angles
        read = n * (Hq + Hkv) * D * 2 + stored * D * 2 + n * c["rot"] * 4
        wrote = n * Hq * D * 2 + stored * 2 * D * (1 if c["fp8"] else 2) + (n * Hkv * D * 2 if c["op"] == "prefill" else 0)
        return {"bytes": read + wrote, "flops": 3 * n * (Hq + Hkv) * c["rot"]}
    if c["op"] == "decode":
        lens = _seq_lens(c)
        rows = int(lens.sum()) * c["full"] + int(np.minimum(lens, c["sink"] + c["window"]).sum()) * (Hkv - c["full"])
        return {"bytes": rows * 2 * D * (1 if c["fp8"] else 2) + c["seqs"] * Hq * D * 4, "flops": 4 * D * rows * (Hq // Hkv)}
    lq, lk = _doc_lens(c)
    pairs = [0, 0]  # visible (query, key) pairs of a compressed and of a full head
    for a, b in zip(lq.tolist(), lk.tolist()):
        pos = np.arange(a) + (b - a)
        hi = np.clip(np.maximum(pos + 1, min(c["prefix"], b)), 0, b)
        lo = np.minimum(np.maximum(pos - c["window"] + 1, 0), hi)
        pairs[1] += int(hi.sum())
        pairs[0] += int((hi - lo + np.minimum(c["sink"], lo)).sum())
    G = Hq // Hkv
    visible = G * (pairs[1] * c["full"] + pairs[0] * (Hkv - c["full"]))
    tq, tk = int(lq.sum()), int(lk.sum())
    bytes_ = 2 * D * (2 * tq * Hq + 2 * tk * Hkv) + 4 * tq * Hq
    if c["op"] == "train":  # dout in, dq, dk, dv out
        bytes_ += 2 * D * (2 * tq * Hq + 2 * tk * Hkv)
    return {"bytes": bytes_, "flops": 4 * D * visible * (3.5 if c["op"] == "train" else 1)}


# ---- what a program has in hand before the call ---------------------------------------------------

class State:
    pass


def _randn(shape, g):
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(torch.bfloat16)


def _tokens(n, c, g):
    """q, k, v of n tokens: apart, or slices of one projection's output."""
    Hq, Hkv, D = c["q_heads"], c["kv_heads"], c["head_dim"]
    if c.get("fused"):
        x = _randn((n, Hq + 2 * Hkv, D), g)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return _randn((n, Hq, D), g), _randn((n, Hkv, D), g), _randn((n, Hkv, D), g)


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
    if c["op"] == "prefill":
        pages = -(-c["tokens"] // TILE)
        return np.array([0]), 0, pages, np.arange(pages)[None]
    lens, n = _start_lens(c), c["seqs"]
    room = LOG_ROOM.get(n, 8192)
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


def _ring_row(t, c):
    return torch.where(t < c["sink"], t, c["sink"] + (t - c["sink"]) % c["window"])


def _pools(c, seqs, pages, device=DEV):
    nf, nc, D = int(_full_heads(c).sum()), c["kv_heads"] - int(_full_heads(c).sum()), c["head_dim"]
    rows = -(-(c["sink"] + c["window"]) // TILE) * TILE
    return nf, nc, (nf, pages, 2, TILE, D), (seqs, nc, 2, rows, D)


def prepare(case, seed):
    c, s = dict(case), State()
    s.c = c
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    s.full = _full_heads(c)
    if own:
        import paper_2510_08525_b200.binding as rl
        s.rl = rl
    if c["op"] in ("append", "prefill"):
        lens, s.room, pages, table = _append_plan(c)
        n = len(lens)
        s.lens, s.step = lens, 0
        longest = int(lens.max()) + s.room if c["op"] == "append" else c["tokens"]
        s.table = _device_table(c, longest)
        s.q, s.k, s.v = _tokens(n if c["op"] == "append" else c["tokens"], c, g)
        s.start = _randn((2, int(lens.sum()), Hkv, D), g)  # the rows the cache holds already
        nf, nc, full_shape, ring_shape = _pools(c, n, pages)
        s.q_out = torch.empty(s.q.shape, dtype=torch.bfloat16, device=DEV)
        s.k_out = torch.empty(s.k.shape, dtype=torch.bfloat16, device=DEV)
        kind = torch.float8_e4m3fn if c["fp8"] else torch.bfloat16
        if own:
            shape = (1, Hkv, Hq, D, n, pages, longest, s.full.astype(np.uint8), c["sink"], c["window"])
            size = (rl.rlkv_paged_size_fp8 if c["fp8"] else rl.rlkv_paged_size)(*shape)
            s.buf = torch.empty(size + 1024, dtype=torch.uint8, device=DEV)
            s.buf = s.buf[-s.buf.data_ptr() % 1024:][:size]
            s.handle = _Handle(rl.rlkv_paged_destroy,
                               rl.rlkv_paged_create_fp8(*shape, _scale8(c, 0), _scale8(c, 1), s.buf, size) if c["fp8"]
                               else rl.rlkv_paged_create(*shape, s.buf, size))
            rl.rlkv_paged_set_rotary(s.handle.h, s.table, longest, c["rot"], c["interleaved"])
            nfull, nring = math.prod(full_shape), math.prod(ring_shape)
            each = 1 if c["fp8"] else 2
            s.pool = s.buf[:nfull * each].view(kind).view(full_shape)
            s.ring = s.buf[nfull * each:(nfull + nring) * each].view(kind).view(ring_shape)
            s.slots = None
            if c["op"] == "append":
                _refill(s)
        else:
            s.pool = torch.zeros(full_shape, dtype=torch.float32, device=DEV).to(kind)
            s.ring = torch.zeros(ring_shape, dtype=torch.float32, device=DEV).to(kind)
            s.heads_full = torch.from_numpy(np.flatnonzero(s.full)).to(DEV)
            s.heads_ring = torch.from_numpy(np.flatnonzero(~s.full)).to(DEV)
            s.pages = torch.from_numpy(table).to(DEV)
            s.pos0 = torch.from_numpy(lens).to(DEV) if c["op"] == "append" else torch.arange(c["tokens"], device=DEV)
            s.seq = torch.arange(n, device=DEV) if c["op"] == "append" else torch.zeros(c["tokens"], dtype=torch.int64, device=DEV)
            if c["op"] == "append":  # the start rows go in as they are
                seq = torch.from_numpy(np.repeat(np.arange(n), lens)).to(DEV)
                pos = torch.from_numpy(np.concatenate([np.arange(x) for x in lens])).to(DEV)
                keep = torch.from_numpy(np.concatenate([np.arange(x) for x in lens]) >= np.repeat(lens, lens) - c["window"]).to(DEV) | (pos < c["sink"])
                _store(s, s.start[0].float(), s.start[1].float(), seq, pos, keep)
        return s
    if c["op"] == "decode":
        lens = _seq_lens(c)
        s.lens = lens
        n, top = c["seqs"], int(lens.max())
        s.k, s.v = (_randn((n, top, Hkv, D), g) for _ in range(2))
        s.q = _randn((n, Hq, D), g)
        slopes = _slopes(c) if c["bias"] else None
        if own:
            pages = int((-(-lens // TILE)).sum())
            shape = (1, Hkv, Hq, D, n, pages, top, s.full.astype(np.uint8), c["sink"], c["window"])
            s.handle = _Handle(rl.rlkv_paged_destroy, rl.rlkv_paged_create_fp8(*shape, _scale8(c, 0), _scale8(c, 1)) if c["fp8"]
                               else rl.rlkv_paged_create(*shape))
            s.slots = np.array([rl.rlkv_paged_seq_open(s.handle.h) for _ in range(n)], np.int32)
            for i in range(n):
                rl.rlkv_paged_prefill(s.handle.h, 0, int(s.slots[i]), s.k[i], s.v[i], int(lens[i]))
            rl.rlkv_paged_set_output_bf16(s.handle.h, 1)
            rl.rlkv_paged_set_scores(s.handle.h, c["cap"], slopes)
            s.out = torch.empty((n, Hq, D), dtype=torch.bfloat16, device=DEV)
            del s.k, s.v
        else:
            if c["fp8"]:
                s.k, s.v = _codes(s.k.float(), _scale8(c, 0)), _codes(s.v.float(), _scale8(c, 1))
                s.k_scale, s.v_scale = (torch.from_numpy(_scale8(c, w)).to(DEV)[:, None] for w in (0, 1))
            s.n = torch.from_numpy(lens).to(DEV)
            s.head_full = torch.from_numpy(s.full).to(DEV)
            s.slopes = torch.from_numpy(slopes).to(DEV) if c["bias"] else None
        return s
    lq, lk = _doc_lens(c)
    starts_q, starts_k = (np.concatenate([[0], np.cumsum(x)]).astype(np.int32) for x in (lq, lk))
    tq, tk = int(lq.sum()) + c["pad"], max(1, int(lk.sum()) + c["pad"])
    s.q = _randn((tq, Hq, D), g)
    kv = _randn((tk, 2 * Hkv, D), g)
    s.k, s.v = kv[:, :Hkv], kv[:, Hkv:]
    s.q_starts = torch.from_numpy(starts_q).to(DEV)
    s.k_starts = torch.from_numpy(starts_k).to(DEV) if c["context"] else None
    s.prefix = torch.full((c["docs"],), c["prefix"], dtype=torch.int32, device=DEV) if c["prefix"] else None
    slopes = _slopes(c) if c["bias"] else None
    s.dout = _randn((tq, Hq, D), g) if c["op"] == "train" else None
    if own:
        s.handle = _Handle(rl.rlkv_prompt_destroy,
                           rl.rlkv_prompt_create(1, Hkv, Hq, D, tq, s.full.astype(np.uint8), c["sink"], c["window"], c["cap"], slopes))
        s.out = torch.zeros((tq, Hq, D), dtype=torch.bfloat16, device=DEV)
        s.lse = torch.zeros((tq, Hq), dtype=torch.float32, device=DEV)
        if c["op"] == "train":
            s.dq, s.dk, s.dv = (torch.zeros(x.shape, dtype=torch.bfloat16, device=DEV) for x in (s.q, s.k, s.v))
    else:
        s.head_full = torch.from_numpy(s.full).to(DEV)
        s.slopes = torch.from_numpy(slopes).to(DEV) if c["bias"] else None
        s.doc_q, s.doc_k, s.pos_q, s.pos_k, s.hi = _doc_indices(c, tq, tk, DEV)
    return s


class _Handle:
    """A handle of the library, given back when the state goes."""

    def __init__(self, destroy, h):
        self.destroy, self.h = destroy, h

    def __del__(self):
        self.destroy(self.h)


def _refill(s):
    """The sequences of an append case at their start lengths: at first, and when a slot has no room left."""
    rl, h = s.rl, s.handle.h
    if s.slots is not None:
        for x in s.slots:
            rl.rlkv_paged_seq_close(h, int(x))
    s.slots = np.array([rl.rlkv_paged_seq_open(h) for _ in s.lens], np.int32)
    at = 0
    for x, n in zip(s.slots, s.lens):
        rl.rlkv_paged_prefill(h, 0, int(x), s.start[0, at:at + n], s.start[1, at:at + n], int(n))
        at += n
    s.step = 0


def _doc_indices(c, tq, tk, device):
    """Document and position of every query and key (-1 and -2: in none), and the first position past
    what a query sees."""
    lq, lk = _doc_lens(c)
    d = np.arange(c["docs"])
    doc_q, doc_k = (np.concatenate([np.repeat(d, x), np.full(t - int(x.sum()), f)]) for x, t, f in ((lq, tq, -1), (lk, tk, -2)))
    pos_q = np.concatenate([np.arange(a) + (b - a) for a, b in zip(lq, lk)] + [np.zeros(tq - int(lq.sum()))])
    pos_k = np.concatenate([np.arange(b) for b in lk] + [np.zeros(tk - int(lk.sum()))])
    return tuple(torch.from_numpy(x.astype(np.int64)).to(device) for x in (doc_q, doc_k, pos_q, pos_k, np.maximum(pos_q + 1, c["prefix"])))


# ---- one pass -------------------------------------------------------------------------------------

def run(s):
    return {"append": _append, "prefill": _append, "decode": _decode, "prompt": _prompt, "train": _prompt}[s.c["op"]](s)


def _rotate(x, cos, sin, c):
    """x [tokens][heads][dim] with its first `rot` elements rotated pairwise."""
    r, cos, sin = c["rot"], cos[:, None], sin[:, None]
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([turned, x[..., r:]], -1)


def _store(s, k, v, seq, pos, keep):
    """K and V rows of tokens `pos` of sequences `seq` into the pages and, where `keep`, into the rings."""
    c = s.c
    if c["fp8"]:
        k, v = _codes(k, _scale8(c, 0)), _codes(v, _scale8(c, 1))
        bits = lambda x: x.view(torch.uint8)  # noqa: E731
    else:
        k, v = k.to(torch.bfloat16), v.to(torch.bfloat16)
        bits = lambda x: x  # noqa: E731
    page = s.pages[seq, pos // TILE]
    for pool, heads, at, row, of in ((s.pool, s.heads_full, page, pos, slice(None)),
                                     (s.ring, s.heads_ring, None, _ring_row(pos, c), keep)):
        if heads.numel() == 0:
            continue
        kk, vv = bits(k)[of][:, heads], bits(v)[of][:, heads]
        h = torch.arange(heads.numel(), device=DEV)[None]
        row = row[of][:, None]
        if at is None:  # [sequence][head][K|V][rows][dim]
            i0, i1 = seq[of][:, None], h
        else:           # [head][page][K|V][rows][dim]
            i0, i1 = h, at[:, None]
        mem = bits(pool)
        if c["fp8"]:    # tiles of 64 rows of K codes and the V codes of the same rows transposed
            t = mem.view(mem.shape[0], mem.shape[1], -1, 2, TILE * c["head_dim"])
            tile = row // TILE if at is None else torch.zeros_like(row)
            t[:, :, :, 0].unflatten(-1, (TILE, c["head_dim"]))[i0, i1, tile, row % TILE] = kk
            t[:, :, :, 1].unflatten(-1, (c["head_dim"], TILE)).transpose(-1, -2)[i0, i1, tile, row % TILE] = vv
        else:
            row = row if at is None else row % TILE
            mem[:, :, 0][i0, i1, row] = kk
            mem[:, :, 1][i0, i1, row] = vv


def _append(s):
    c = s.c
    if own:
        rl, h = s.rl, s.handle.h
        if c["op"] == "append":
            if s.step == s.room:
                _refill(s)
            s.step += 1
            rl.rlkv_paged_append_rotated(h, 0, s.slots, s.q, s.k, s.v, s.q_out)
            return {"q": s.q_out, "pool": s.pool, "ring": s.ring}
        slot = rl.rlkv_paged_seq_open(h)
        rl.rlkv_paged_prefill_rotated(h, 0, slot, s.q, s.k, s.v, c["tokens"], s.q_out, s.k_out)
        rl.rlkv_paged_seq_close(h, slot)
        return {"q": s.q_out, "k": s.k_out, "pool": s.pool, "ring": s.ring}
    pos = s.pos0 + s.step
    if c["op"] == "append":
        s.step = (s.step + 1) % s.room
        keep = torch.ones_like(pos, dtype=torch.bool)
    else:
        keep = (pos < c["sink"]) | (pos >= c["tokens"] - c["window"])
    cos, sin = s.table[pos].unbind(-1)
    q = _rotate(s.q.float(), cos, sin, c).to(torch.bfloat16)
    k = _rotate(s.k.float(), cos, sin, c)
    _store(s, k, s.v.float(), s.seq, pos, keep)
    out = {"q": q, "pool": s.pool, "ring": s.ring}
    return out if c["op"] == "append" else {**out, "k": k.to(torch.bfloat16)}


def _scores(x, c, slopes, dist):
    """Capped and biased scores of x = q.k / sqrt(dim); `slopes` and `dist` broadcast against x."""
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    return x if slopes is None else x - slopes * dist


def _decode(s):
    c = s.c
    if own:
        s.rl.rlkv_paged_decode_attention(s.handle.h, 0, s.slots, s.q, s.out)
        return s.out
    n, Hkv, D = c["seqs"], c["kv_heads"], c["head_dim"]
    k, v = s.k.float(), s.v.float()
    if c["fp8"]:
        k, v = k * s.k_scale, v * s.v_scale
    q = s.q.float().view(n, Hkv, -1, D)
    x = torch.matmul(q, k.permute(0, 2, 3, 1)) / math.sqrt(D)          # [seq][kv head][group][token]
    t = torch.arange(k.shape[1], device=DEV)
    dist = (s.n[:, None] - 1 - t)[:, None, None]
    x = _scores(x, c, None if s.slopes is None else s.slopes.view(1, Hkv, -1, 1), dist)
    seen = (dist >= 0) & (s.head_full.view(1, -1, 1, 1) | (t < c["sink"]) | (dist < c["window"]))
    x = x.masked_fill(~seen, -math.inf)
    p = (x - x.amax(-1, keepdim=True)).exp()
    o = torch.matmul(p, v.transpose(1, 2)) / p.sum(-1, keepdim=True)
    return o.reshape(n, -1, D).to(torch.bfloat16)


def _prompt(s):
    c = s.c
    train = c["op"] == "train"
    if own:
        rl, h = s.rl, s.handle.h
        rl.rlkv_prompt_attention(h, 0, s.q, s.k, s.v, s.q_starts, s.k_starts, s.prefix, s.out, s.lse)
        if not train:
            return {"out": s.out, "lse": s.lse}
        rl.rlkv_prompt_attention_backward(h, 0, s.q, s.k, s.v, s.q_starts, s.k_starts, s.prefix, s.out, s.lse, s.dout, s.dq, s.dk, s.dv)
        return {"out": s.out, "lse": s.lse, "dq": s.dq, "dk": s.dk, "dv": s.dv}
    D, Hkv, scale = c["head_dim"], c["kv_heads"], 1 / math.sqrt(c["head_dim"])
    heads = lambda x: x.float().transpose(0, 1).unflatten(0, (Hkv, -1))  # noqa: E731  [kv head][group][token][dim]
    back = lambda x: x.flatten(0, 1).transpose(0, 1).to(torch.bfloat16).contiguous()  # noqa: E731
    q, k, v = heads(s.q), heads(s.k), heads(s.v)
    dist = s.pos_q[:, None] - s.pos_k
    seen = (s.doc_q[:, None] == s.doc_k) & (s.pos_k < s.hi[:, None])
    seen = seen & (s.head_full.view(-1, 1, 1, 1) | (s.pos_k < c["sink"]) | (dist < c["window"]))
    x = _scores(torch.matmul(q, k.transpose(-1, -2)).mul_(scale), c, None if s.slopes is None else s.slopes.view(Hkv, -1, 1, 1), dist.abs())
    slope_of_cap = None
    if train and c["cap"]:  # 1 - tanh^2, from the capped score itself
        y = x if s.slopes is None else x + s.slopes.view(Hkv, -1, 1, 1) * dist.abs()
        slope_of_cap = 1 - (y / c["cap"]) ** 2
    x = x.masked_fill(~seen, -math.inf)
    m = x.amax(-1, keepdim=True)
    p = (x - torch.where(m == -math.inf, 0.0, m)).exp()
    del x
    total = p.sum(-1, keepdim=True)
    p = p.div_(torch.where(total == 0, 1.0, total))
    o = torch.matmul(p, v)
    lse = (m + total.log()).squeeze(-1).flatten(0, 1).T
    lse = torch.where(s.doc_q[:, None] < 0, 0.0, lse).contiguous()
    if not train:
        return {"out": back(o), "lse": lse}
    do = torch.where(s.doc_q[:, None] < 0, 0.0, heads(s.dout))
    dv = torch.matmul(p.transpose(-1, -2), do).sum(1, keepdim=True)
    ds = p.mul_(torch.matmul(do, v.transpose(-1, -2)).sub_((do * o).sum(-1, keepdim=True)))
    if slope_of_cap is not None:
        ds = ds.mul_(slope_of_cap)
    dq = torch.matmul(ds, k) * scale
    dk = torch.matmul(ds.transpose(-1, -2), q).sum(1, keepdim=True) * scale
    return {"out": back(o), "lse": lse, "dq": back(dq), "dk": back(dk), "dv": back(dv)}


# ---- the same in 64 bits, written from the definitions ---------------------------------------------

def exact(case, seed):
    """What run() returns for a new state, head by head and sequence by sequence in 64 bits."""
    c = dict(case)
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    if c["op"] in ("append", "prefill"):
        return _exact_append(c, g)
    return _exact_decode(c, g) if c["op"] == "decode" else _exact_prompt(c, g)


def _exact_append(c, g):
    Hq, Hkv, D, r = c["q_heads"], c["kv_heads"], c["head_dim"], c["rot"]
    prefill = c["op"] == "prefill"
    lens, _, pages, table = _append_plan(c)
    q, k, v = _tokens(c["tokens"] if prefill else len(lens), c, g)
    start = _randn((2, int(lens.sum()), Hkv, D), g).double()
    nf, nc, full_shape, ring_shape = _pools(c, len(lens), pages)
    pos = torch.arange(c["tokens"]) if prefill else torch.from_numpy(lens)
    angle = (pos.double()[:, None] * torch.from_numpy(_inv_freq(c))).to(DEV)
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def rotated(x):
        x = x.double().clone()
        first, second = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
        z = torch.complex(first.contiguous(), second.contiguous()) * turn
        first.copy_(z.real)
        second.copy_(z.imag)
        return x

    q, k, v = rotated(q), rotated(k), v.double()
    if math.prod(full_shape) > 1 << 29:  # too large to hold in 64 bits
        return {"q": q, "pool": None, "ring": None, "k": k} if prefill else {"q": q, "pool": None, "ring": None}
    pool = torch.zeros(full_shape, dtype=torch.float64, device=DEV)
    ring = torch.zeros(ring_shape, dtype=torch.float64, device=DEV)
    full = _full_heads(c)
    at = 0
    for i in range(len(lens)):
        n0 = int(lens[i])
        rows = [torch.cat([start[w, at:at + n0], x if prefill else x[i:i + 1]]) for w, x in ((0, k), (1, v))]
        at += n0
        n = rows[0].shape[0]
        t = torch.arange(n, device=DEV)
        page = torch.from_numpy(table[i]).to(DEV)[t // TILE]
        last = t[(t < c["sink"]) | (t >= n - c["window"])]
        for w in (0, 1):
            # an 8-bit cache is compared in units of its scale
            x = rows[w] / torch.from_numpy(_scale8(c, w)).to(DEV).double()[:, None] if c["fp8"] else rows[w]
            for f, h in enumerate(np.flatnonzero(full)):
                pool[f, page, w, t % TILE] = x[:, h]
            for f, h in enumerate(np.flatnonzero(~full)):
                ring[i, f, w, _ring_row(last, c)] = x[last, h]
    if c["fp8"]:  # tiles of K codes and transposed V codes
        pool = torch.stack([pool[:, :, 0].flatten(-2), pool[:, :, 1].transpose(-1, -2).flatten(-2)], 2).view(full_shape)
        tiles = ring.unflatten(3, (-1, TILE))
        ring = torch.stack([tiles[:, :, 0].flatten(-2), tiles[:, :, 1].transpose(-1, -2).flatten(-2)], 3).reshape(ring_shape)
    out = {"q": q, "pool": pool, "ring": ring}
    return {**out, "k": k} if prefill else out


def _exact_decode(c, g):
    D, Hq, Hkv = c["head_dim"], c["q_heads"], c["kv_heads"]
    lens, full, G = _seq_lens(c), _full_heads(c), c["q_heads"] // c["kv_heads"]
    top = int(lens.max())
    k, v = (_randn((c["seqs"], top, Hkv, D), g) for _ in range(2))
    q = _randn((c["seqs"], Hq, D), g).double()
    out = torch.empty((c["seqs"], Hq, D), dtype=torch.float64, device=DEV)
    for i in range(c["seqs"]):
        n = int(lens[i])
        t = torch.arange(n, device=DEV)
        kept = t[(t < c["sink"]) | (t >= n - c["window"])]
        for h in range(Hkv):
            of = t if full[h] else kept
            kk, vv = k[i, :n, h][of], v[i, :n, h][of]
            if c["fp8"]:
                kk, vv = (_codes(x.float()[:, None], _scale8(c, w)[h:h + 1])[:, 0].double() * float(_scale8(c, w)[h])
                          for w, x in ((0, kk), (1, vv)))
            x = q[i, h * G:(h + 1) * G] @ kk.double().T / math.sqrt(D)
            if c["cap"]:
                x = c["cap"] * torch.tanh(x / c["cap"])
            if c["bias"]:
                x = x - torch.from_numpy(_slopes(c)).to(DEV).double()[h * G:(h + 1) * G, None] * (n - 1 - of)
            out[i, h * G:(h + 1) * G] = torch.softmax(x, -1) @ vv.double()
    return out


def _exact_prompt(c, g):
    D, Hq, Hkv, train = c["head_dim"], c["q_heads"], c["kv_heads"], c["op"] == "train"
    G, scale, full = Hq // Hkv, 1 / math.sqrt(D), _full_heads(c)
    lq, lk = _doc_lens(c)
    tq, tk = int(lq.sum()) + c["pad"], max(1, int(lk.sum()) + c["pad"])
    q = _randn((tq, Hq, D), g).double()
    kv = _randn((tk, 2 * Hkv, D), g).double()
    k, v = kv[:, :Hkv], kv[:, Hkv:]
    dout = _randn((tq, Hq, D), g).double() if train else None
    zeros = lambda x: torch.zeros(x.shape, dtype=torch.float64, device=DEV)  # noqa: E731
    out, lse = zeros(q), torch.zeros((tq, Hq), dtype=torch.float64, device=DEV)
    dq, dk, dv = (zeros(x) for x in (q, k, v)) if train else (None,) * 3
    slopes = _slopes(c)
    q0 = k0 = 0
    for a, b in zip(lq.tolist(), lk.tolist()):
        rows, keys = slice(q0, q0 + a), slice(k0, k0 + b)
        q0, k0 = q0 + a, k0 + b
        i, j = torch.arange(a, device=DEV)[:, None] + (b - a), torch.arange(b, device=DEV)
        causal = (j <= i) | (j < c["prefix"])
        local = causal & ((j < c["sink"]) | (i - j < c["window"]))
        for h in range(Hq):
            kh, vh, qh = k[keys, h // G], v[keys, h // G], q[rows, h]
            y = qh @ kh.T * scale
            if c["cap"]:
                tanh = torch.tanh(y / c["cap"])
                y = c["cap"] * tanh
            if c["bias"]:
                y = y - float(slopes[h]) * (i - j).abs()
            y = y.masked_fill(~(causal if full[h // G] else local), -math.inf)
            l = torch.logsumexp(y, -1) if b else torch.full((a,), -math.inf, dtype=torch.float64, device=DEV)
            lse[rows, h] = l
            p = (y - torch.where(l == -math.inf, 0.0, l)[:, None]).exp()
            out[rows, h] = p @ vh
            if train:
                do = dout[rows, h]
                dv[keys, h // G] += p.T @ do
                ds = p * (do @ vh.T - (do * out[rows, h]).sum(-1, keepdim=True))
                if c["cap"]:
                    ds = ds * (1 - tanh * tanh)
                dq[rows, h] = ds @ kh * scale
                dk[keys, h // G] += ds.T @ qh * scale
    res = {"out": out, "lse": lse}
    return {**res, "dq": dq, "dk": dk, "dv": dv} if train else res
