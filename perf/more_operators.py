"""Timed cases of the operators by which sequences live on in a paged KV cache: attention over first tokens and a window, and
blocks that are shared, copied, given back and moved together.

  sinks    tutti_kv_attend_sinks: attention over what a sequence holds, causal, of the last `window` tokens and the `sinks` first
           ones; the blocks between them need not be in the table any more.
  fork     tutti_blocks_fork: sequences that go on from another's blocks: its table entries shared, the last block as a copy of
           one's own, and new blocks where a sequence grows.  d_uses counts the table entries that name a block.
  free     tutti_blocks_free: table entries, and the blocks that nobody else names, given back.
  compact  tutti_blocks_compact: the blocks in use become the first ones of the pool, the last of them first; tables follow.
  copy     tutti_blocks_copy: one layer's keys and values (codes and scales) of the blocks that were copied or moved.

`own` chooses between the plain form in elementary torch operations and the framework's calls.  Fork, free and compact change
their counts and tables, so a pass first puts these back, with one copy, on either side: passes are alike.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
FLOOR = -64                  # exponent of the smallest scale of an 8-bit block
NONE = -1                    # a table entry that names no block
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}

# T: tokens a block; h: KV heads; hq: query heads; d: head size; cache: type of the pool; x: type of queries and outputs
SINKS = dict(op="sinks", T=16, h=8, hq=32, d=128, x="bf16", cache="bf16", hnd=False, seqs=1, new=1, new_spread=False, held=1024,
             held_spread="even", window=256, sinks=4)
# blocks: of the pool; groups: requests; beams: sequences of a request, which share their first blocks; row: blocks a sequence
# has on average, with those of the others in its group; gone: share of the requests that have ended (their blocks are free again)
TABLE = dict(op="fork", blocks=65536, groups=4, beams=4, row=64, spread=True, gone=0.25)
COPY = dict(op="copy", T=16, h=8, d=128, cache="bf16", hnd=False, pairs=4, blocks=4096)


def _sinks(name, **kw):
    return dict(SINKS, name=name, **kw)


def _table(name, **kw):
    return dict(TABLE, name=name, **kw)


def _copy(name, **kw):
    return dict(COPY, name=name, **kw)


def listed():
    return [
        # a one-layer model of 2 heads x 64 far beyond its window: latency
        _sinks("sinks_tiny", h=2, hq=4, d=64, x="fp16", cache="fp16", held=1500, window=256),
        # 8B shape, 64 endless streams of uneven age, 8-bit cache: 4 first tokens and 4,096 last ones of each
        _sinks("sinks_decode_64_e4m3", seqs=64, new=64, held=60000, held_spread="zipf", cache="e4m3", window=4096),
        # a chunk of a long document: 2,048 tokens behind 30,000, 64 first tokens beside the window
        _sinks("sinks_chunk_2k_behind_30k", new=2048, held=32048, window=4096, sinks=64),
        # 5 heads x 80, head-major 8-bit pool: a prompt's chunk and decoding streams in one step, an odd window
        _sinks("sinks_mixed_5x80_e4m3", h=5, hq=20, d=80, x="fp16", cache="e4m3", hnd=True, T=32, seqs=12, new=1511,
               new_spread="one", held=9000, held_spread="zipf", window=1001, sinks=20),
        # a step of beam search, one request: 4 beams of 64 blocks go on from others' tables; the smallest call
        _table("fork_beams_4", groups=1, beams=4, row=64),
        # parallel sampling in a large pool: 128 requests x 8 samples with long shared prompts
        _table("fork_samples_1024", blocks=1 << 20, groups=128, beams=8, row=512),
        # streams past their window: each of 256 gives back the block that has just left it
        _table("free_window_256", op="free", groups=256, beams=1, row=200),
        # a serving batch ends: 96 requests of 4 samples, long tables, most of their entries shared
        _table("free_batch_384", op="free", blocks=1 << 19, groups=96, beams=4, row=2000),
        # 8B pool of 65,536 blocks, a third of the requests have ended
        _table("compact_8b", op="compact", groups=160, beams=2, row=200, gone=0.33),
        # a pool of a million blocks after a burst: half of the requests have ended
        _table("compact_1m", op="compact", blocks=1 << 20, groups=1000, beams=1, row=900, gone=0.5),
        # what a step of beam search copies of a layer: 3 blocks of 32 KiB and their values'
        _copy("copy_beams_3", pairs=3),
        # what compaction moves of a layer: 6,001 blocks, e4m3 with their scales
        _copy("copy_compact_6k_e4m3", pairs=6001, blocks=16384, cache="e4m3", T=32),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("sinks", "sinks", "sinks", "fork", "free", "compact", "copy"))
    if op == "copy":
        case = dict(COPY, T=rng.choice((16, 16, 32, 64)), h=rng.choice((1, 2, 5, 8)), d=rng.choice((64, 80, 128, 128)),
                    cache=rng.choice(("bf16", "fp16", "e4m3")), hnd=rng.random() < 0.3)
        case["blocks"] = min(16384, (1 << 30) // (case["T"] * case["h"] * case["d"] * 2))
        return dict(case, pairs=_log(rng, 1, min(6000, case["blocks"] // 2)))
    if op != "sinks":
        blocks = _log(rng, 4096, 1 << 20)
        beams = rng.choice((1, 2, 3, 4, 8))
        row = _log(rng, 2, min(2000, blocks // 8))
        groups = _log(rng, 1, max(1, min(1024 // beams, blocks // (2 * row + 5 * beams))))
        return dict(TABLE, op=op, blocks=blocks, groups=groups, beams=beams, row=row, spread=rng.random() < 0.7,
                    gone=rng.choice((0.0, 0.1, 0.3, 0.5)))
    while True:
        h, group = rng.choice((1, 2, 4, 5, 8, 8)), rng.choice((1, 2, 4, 4, 5, 8))
        if h * group <= 64:
            break
    x = rng.choice(("bf16", "bf16", "fp16"))
    case = dict(SINKS, T=rng.choice((16, 16, 32, 64)), h=h, hq=h * group, d=rng.choice((64, 80, 96, 112, 128, 128)), x=x,
                cache=rng.choice((x, "e4m3")), hnd=rng.random() < 0.3, held_spread=rng.choice(("even", "zipf")),
                window=_log(rng, 60, 8192), sinks=_log(rng, 1, 128))
    kind = rng.choice(("decode", "decode", "verify", "prompt", "mixed"))
    if kind in ("decode", "verify"):
        seqs = _log(rng, 1, 128)
        each = 1 if kind == "decode" else rng.randint(2, 8)
        case["window"] = min(case["window"], 2000000 // (seqs * h))
        return dict(case, seqs=seqs, new=seqs * each, held=_log(rng, each, 100000))
    seqs = _log(rng, 1, 8) if kind == "prompt" else rng.randint(3, 12)
    padded = h * group * (seqs if kind == "mixed" else 1)
    new = max(seqs, _log(rng, 64, min(3000, math.isqrt(600000000 // padded))))
    most = 600000000 // (padded * new)                                           # keys for the scores of the plain form
    case["window"] = max(60, min(case["window"], most - new))
    return dict(case, seqs=seqs, new=new, new_spread=True if kind == "prompt" else "one",
                held=0 if rng.random() < 0.3 else _log(rng, 64, 30000))


class _State:
    pass


# ---- attention: what a case's sequences look like, the same for every seed (they decide the outputs' sizes)

def _shares(total, n, spread, rng):
    """n whole numbers of at least 1 that add up to total."""
    if spread == "one":           # one large, the others 1
        return np.array([total - (n - 1)] + [1] * (n - 1))
    w = rng.uniform(0.2, 1.0, n) if spread else np.ones(n)
    got = 1 + np.floor(w / w.sum() * (total - n)).astype(np.int64)
    got[np.argsort(-w, kind="stable")[:total - int(got.sum())]] += 1
    return got


def _sequences(case):
    """(new tokens, tokens held in all with the new ones) of each sequence."""
    n = case["seqs"]
    rng = np.random.default_rng(20260504)
    new = _shares(case["new"], n, case["new_spread"], rng)
    if case["held_spread"] == "zipf":     # lengths over 64 ranks, as a mix of long and short contexts has them
        ranks = np.arange(1, 65, dtype=np.float64)
        p = ranks ** -1.1
        w = rng.choice(ranks, size=n, p=p / p.sum()) * rng.uniform(0.3, 1.0, size=n)
        held = np.floor(case["held"] * np.minimum(w / w.mean(), 5.0)).astype(np.int64)
    else:
        held = np.full(n, case["held"], np.int64) - np.arange(n) % 7 * (1 if n > 1 else 0)
    return new, np.maximum(held, new) if case["held"] else new


def _first_key(case, new, held):
    """Of the window of the first new token."""
    return np.maximum(0, held - new + 1 - case["window"])


def _plane(case, blocks):
    return (blocks, case["h"], case["T"], case["d"]) if case["hnd"] else (blocks, case["T"], case["h"], case["d"])


def _quantised(x, token_dim, scale_floats):
    """e4m3 values of x [blocks, ., ., d] and the scales [blocks, scale_floats] of its blocks and heads."""
    top = x.abs().amax(dim=(token_dim, 3))
    m, e = torch.frexp(top)
    scale = torch.ldexp(torch.ones_like(top), torch.clamp(e - 9 + (m > 0.875).int(), min=FLOOR))
    codes = (x / scale.unsqueeze(token_dim).unsqueeze(3)).to(torch.float8_e4m3fn)
    padded = torch.zeros(top.shape[0], scale_floats, device=DEV)
    padded[:, :top.shape[1]] = scale
    return codes, padded


def _make_pool(st, case, blocks, gen):
    """What earlier tokens left in the pool: blocks of uneven magnitude, a few large channels in the keys."""
    st.planes, st.scales = [], [None, None]
    for kind in range(2):
        plane = torch.empty(_plane(case, blocks), dtype=TYPES[case["cache"]], device=DEV)
        scales = torch.empty(blocks, -(-case["h"] // 4) * 4, device=DEV)
        loud = torch.ones(case["d"], device=DEV)
        if kind == 0:
            loud[torch.randint(0, case["d"], (3,), generator=gen, device=DEV)] = 4.0
        step = max(1, (1 << 27) // (case["T"] * case["h"] * case["d"]))
        for lo in range(0, blocks, step):
            hi = min(blocks, lo + step)
            v = torch.randn(_plane(case, hi - lo), generator=gen, device=DEV) * loud
            v *= torch.exp(0.3 * torch.randn(hi - lo, 1, 1, 1, generator=gen, device=DEV))
            if case["cache"] == "e4m3":
                plane[lo:hi], scales[lo:hi] = _quantised(v, 2 if case["hnd"] else 1, scales.shape[1])
            else:
                plane[lo:hi] = v.to(plane.dtype)
        st.planes.append(plane)
        if case["cache"] == "e4m3":
            st.scales[kind] = scales


def _prepare_sinks(case, seed):
    rng = np.random.default_rng([seed, case["new"], case["held"]])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    T, h, hq, d, n = case["T"], case["h"], case["hq"], case["d"], case["seqs"]
    new, held = _sequences(case)
    st = _State()
    st.rows = int(new.sum())
    st.max_new = int(new.max())
    need = -(-held // T)
    off = np.cumsum(need) - need
    # blocks that some query sees are there, those between the first tokens and the window have been given back
    number = np.arange(int(need.sum())) - np.repeat(off, need)
    live = (number * T < case["sinks"]) | ((number + 1) * T > np.repeat(_first_key(case, new, held), need))
    blocks = int(live.sum()) + int(live.sum()) // 8 + 3
    table = np.full(live.size, NONE, np.int32)
    table[live] = rng.permutation(blocks)[:int(live.sum())]
    row0 = np.cumsum(new) - new
    st.blocks = blocks
    st.table = torch.from_numpy(table).to(DEV)
    st.seqs = torch.from_numpy(np.stack([row0, new, held, off], 1).astype(np.int32)).to(DEV)
    _make_pool(st, case, blocks, gen)
    # one projection gives queries, keys and values side by side, as a fused product leaves them
    x = TYPES[case["x"]]
    st.q = torch.randn(st.rows, hq + 2 * h, d, generator=gen, device=DEV).to(x)[:, :hq]
    st.out = torch.empty(st.rows, hq, d, dtype=x, device=DEV)
    st.lse = torch.empty(st.rows, hq, device=DEV)
    # keys that a sequence's queries see at most, for the plain form's gather
    first = _first_key(case, new, held)
    st.most_keys = int((held - first + np.minimum(case["sinks"], first)).max())
    return st


# ---- tables

def _rows_of(case):
    """Blocks of each sequence, and how many of them its group shares."""
    rng = np.random.default_rng(20260505)
    groups, beams = case["groups"], case["beams"]
    n = case["row"] * rng.uniform(0.3, 1.7, groups) if case["spread"] else np.full(groups, float(case["row"]))
    n = np.maximum(1, n.astype(np.int64))
    shared = np.where(beams > 1, np.maximum(0, n - rng.integers(1, 6, groups)), 0)
    return np.repeat(n, beams), np.repeat(shared, beams)


def _records(case):
    """Fork: (source, n_shared, n_copied, n_new) of each sequence that goes on; a sequence's first child keeps its last block, the
    others get a copy, and every few sequences begin a new block."""
    rng = np.random.default_rng(20260506)
    n, _ = _rows_of(case)
    beams = case["beams"]
    i = np.arange(n.size)
    source = i // beams * beams + (rng.integers(0, beams, n.size) if beams > 1 else 0)
    first = np.ones(n.size, bool)
    order = np.argsort(source, kind="stable")
    first[order[1:]] = source[order][1:] != source[order][:-1]
    copied = np.where(first, 0, 1)
    return source, n - copied, copied, (rng.random(n.size) < 1 / 8).astype(np.int64)


def _ended(case):
    """Requests that have ended, in compaction: which sequences."""
    rng = np.random.default_rng(20260507)
    return np.repeat(rng.random(case["groups"]) < case["gone"], case["beams"])


def _distinct(case):
    """Blocks that the sequences name in all."""
    n, shared = _rows_of(case)
    beams = case["beams"]
    return int((n - shared).sum() + shared[::beams].sum())


def _prepare_table(case, seed):
    rng = np.random.default_rng([seed, case["blocks"], case["row"]])
    n, shared = _rows_of(case)
    beams, width = case["beams"], int(n.max()) + 1
    st = _State()
    st.blocks, st.width = case["blocks"], width
    need = _distinct(case)
    # blocks that other requests hold lie among these, as an engine that has run for a while leaves them
    held = rng.permutation(case["blocks"])[:min(case["blocks"], need + case["blocks"] // 8)].astype(np.int32)
    mine, others = held[:need], held[need:]
    halves = 2 if case["op"] == "fork" else 1
    table = np.full((halves, n.size, width), NONE, np.int32)
    at = 0
    for i in range(n.size):
        if i % beams == 0:
            prefix = mine[at:at + shared[i]]
            at += int(shared[i])
        table[0, i, :shared[i]] = prefix
        table[0, i, shared[i]:n[i]] = mine[at:at + n[i] - shared[i]]
        at += int(n[i] - shared[i])
    if case["op"] == "compact":
        table[0, _ended(case)] = NONE
    uses = np.bincount(table[table >= 0], minlength=case["blocks"]).astype(np.int32)
    uses[others] = 1
    st.saved = torch.from_numpy(np.concatenate([uses, table.ravel()])).to(DEV)
    st.live = torch.empty_like(st.saved)
    st.uses, st.table = st.live.split([case["blocks"], table.size])
    row = np.arange(n.size) * width
    if case["op"] == "fork":
        source, n_shared, n_copied, n_new = _records(case)
        rec = np.zeros((n.size, 8), np.int32)
        rec[:, 0], rec[:, 1] = source * width, n.size * width + row
        rec[:, 2], rec[:, 3], rec[:, 4] = n_shared, n_copied, n_new
        st.max_entries, st.total = int((n_shared + n_copied + n_new).max()), int((n_shared + n_copied + n_new).sum())
        st.max_pairs = max(1, int(n_copied.sum()))
        st.records = torch.from_numpy(rec).to(DEV)
    elif case["op"] == "free":
        # one request's samples: all of their entries; streams: the block that has left the window
        first, count = (np.zeros_like(n), n) if beams > 1 else (np.minimum(1, n - 1), np.ones_like(n))
        st.max_entries, st.total = int(count.max()), int(count.sum())
        st.records = torch.from_numpy(np.stack([row + first, count], 1).astype(np.int32)).to(DEV)
    else:
        st.max_pairs = case["blocks"] // 2
    if case["op"] != "free":
        st.pairs = torch.full((st.max_pairs, 2), NONE, dtype=torch.int32, device=DEV)
        st.totals = torch.zeros(2 if case["op"] == "compact" else 1, dtype=torch.int32, device=DEV)
    return st


def _prepare_copy(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    st = _State()
    st.blocks = case["blocks"]
    _make_pool(st, case, case["blocks"], gen)
    order = torch.randperm(case["blocks"], generator=gen, device=DEV)[:2 * case["pairs"]].to(torch.int32)
    st.pairs = order.view(2, -1).T.contiguous()
    return st


def prepare(case, seed):
    make = {"sinks": _prepare_sinks, "copy": _prepare_copy}.get(case["op"], _prepare_table)
    st = make(case, seed)
    st.case, st.handles = case, None
    return st


# ---- the framework's calls

def _pool(st, B):
    c = st.case
    pool = B.make_pool(st.planes[0], st.planes[1], num_blocks=st.blocks, block_tokens=c["T"], num_kv_heads=c["h"],
                       head_dim=c["d"], elt_bytes=st.planes[0].element_size(),
                       pool_layout=B.LAYOUT_HND if c["hnd"] else B.LAYOUT_NHD)
    return pool, None if st.scales[0] is None else B.make_scales(*st.scales)


def _handles(st):
    """What a program makes once and uses in every step or layer: records of the pool and the batch, work memory."""
    from paper_2605_03375_amd import binding as B
    c = st.case
    h = _State()
    h.B = B
    need = 0
    if c["op"] in ("sinks", "copy"):
        h.pool, h.scales = _pool(st, B)
    if c["op"] == "sinks":
        h.batch = B.make_batch(st.seqs, c["seqs"], st.max_new, st.table, st.table.numel(), st.rows)
        h.attn = B.make_attn(c["hq"], {"bf16": B.BF16, "fp16": B.FP16}[c["x"]], 1.0 / math.sqrt(c["d"]), window=c["window"])
        h.rows = [B.make_rows(t) for t in (st.q, st.out)]
        need = B.tutti_kv_attend_work_bytes(h.pool, h.batch, h.attn)
    elif c["op"] == "fork":
        need = B.tutti_blocks_fork_work_bytes(st.blocks, st.records.shape[0])
    elif c["op"] == "compact":
        need = B.tutti_blocks_compact_work_bytes(st.blocks)
    h.work = torch.empty(need, dtype=torch.uint8, device=DEV)
    return h


def _result(st):
    if st.case["op"] == "sinks":
        return {"out": st.out, "lse": st.lse}
    if st.case["op"] == "copy":
        r = {"k": st.planes[0], "v": st.planes[1]}
        if st.scales[0] is not None:
            r.update(k_scale=st.scales[0], v_scale=st.scales[1])
        return r
    r = {"uses": st.uses, "table": st.table}
    if st.case["op"] != "free":
        r.update(pairs=st.pairs, totals=st.totals)
    return r


def _own(st):
    if st.handles is None:
        st.handles = _handles(st)
    h, op = st.handles, st.case["op"]
    B = h.B
    if op == "sinks":
        B.tutti_kv_attend_sinks(h.pool, h.scales, h.batch, h.attn, st.case["sinks"], *h.rows, st.lse, h.work, h.work.numel())
    elif op == "copy":
        B.tutti_blocks_copy(h.pool, h.scales, st.pairs, None, st.pairs.shape[0])
    elif op == "fork":
        B.tutti_blocks_fork(st.uses, st.blocks, st.table, st.table.numel(), st.records, st.records.shape[0], st.max_entries,
                            st.pairs, st.totals, st.max_pairs, h.work, h.work.numel())
    elif op == "free":
        B.tutti_blocks_free(st.uses, st.blocks, st.table, st.table.numel(), st.records, st.records.shape[0], st.max_entries)
    else:
        B.tutti_blocks_compact(st.uses, st.blocks, st.table, st.table.numel(), st.pairs, st.totals, st.max_pairs, h.work,
                               h.work.numel())
    return _result(st)


# ---- the plain form

def _sinks_plain(st):
    c = st.case
    T, h, hq, d, n = c["T"], c["h"], c["hq"], c["d"], c["seqs"]
    row0, new, held, off = st.seqs.long().unbind(1)
    # the keys that a sequence's queries see, gathered: its first tokens, then from the first query's window on
    first = (held - new + 1 - c["window"]).clamp(min=0)
    sinks = first.clamp(max=c["sinks"])
    a = torch.arange(st.most_keys, device=DEV)
    j = torch.where(a < sinks.unsqueeze(1), a, a + (first - sinks).unsqueeze(1))   # [n, keys]
    there = j < held.unsqueeze(1)
    index = torch.where(there, off.unsqueeze(1) + j // T, off.unsqueeze(1))
    block, slot = st.table.long()[index].clamp(min=0), j % T
    keys, values = [], []
    for plane, scales, to in zip(st.planes, st.scales, (keys, values)):
        x = plane.view(torch.int16 if scales is None else torch.uint8)                # (indexed as they lie)
        x = (x.transpose(1, 2) if c["hnd"] else x)[block, slot].view(plane.dtype).float()       # [n, keys, h, d]
        if scales is not None:
            x *= scales[block][..., :h].unsqueeze(3)
        to.append(x.masked_fill_(~there.unsqueeze(2).unsqueeze(3), 0.0).transpose(1, 2).contiguous())
    i = torch.arange(st.max_new, device=DEV)
    q = st.q.float()[(row0.unsqueeze(1) + i).clamp(max=st.rows - 1)]           # [n, new, hq, d]
    q = q.transpose(1, 2).reshape(n, h, hq // h * st.max_new, d)
    scores = torch.matmul(q, keys.pop().transpose(2, 3).contiguous()) * (1.0 / math.sqrt(d))
    scores = scores.view(n, h, hq // h, st.max_new, st.most_keys)
    place = ((held - new).unsqueeze(1) + i).unsqueeze(2)                       # [n, new, 1]
    j = j.unsqueeze(1)
    seen = there.unsqueeze(1) & (j <= place) & ((j > place - c["window"]) | (j < c["sinks"]))
    scores.masked_fill_(~seen.unsqueeze(1).unsqueeze(1), -math.inf)
    top = scores.amax(4, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weights = scores.sub_(top).exp_()
    total = weights.sum(4, keepdim=True)
    out = torch.matmul(weights.view(n, h, -1, st.most_keys), values.pop()).view(n, hq, st.max_new, d)
    out = out / total.view(n, hq, st.max_new, 1)
    lse = (top + total.log()).view(n, hq, st.max_new)
    row = torch.arange(st.rows, device=DEV)
    s = torch.searchsorted(row0 + new, row, right=True)
    st.out.copy_(out[s, :, row - row0[s]])
    st.lse.copy_(lse[s, :, row - row0[s]])


def _ranked(mask):
    """For each true place of the mask its number among them (one behind the last for the others), and how many there are."""
    count = torch.cumsum(mask, 0)
    return torch.where(mask, count - 1, mask.numel()), count[-1]


def _listed_places(mask):
    """The true places of a mask in order, then NONE, as many as the mask has places and one more."""
    rank, n = _ranked(mask)
    places = torch.full((mask.numel() + 1,), NONE, device=DEV)
    places[rank] = torch.arange(mask.numel(), device=DEV)
    return torch.where(torch.arange(mask.numel() + 1, device=DEV) < n, places, NONE), rank, n


def _entries(count, total):
    """For each of `total` entries the record that it belongs to and its place in it."""
    r = torch.repeat_interleave(torch.arange(count.numel(), device=DEV), count, output_size=total)
    return r, torch.arange(total, device=DEV) - (torch.cumsum(count, 0) - count)[r]


def _fork_plain(st):
    src, dst, shared, copied, new = st.records.long().unbind(1)[:5]
    free, _, _ = _listed_places(st.uses == 0)
    r, place = _entries(shared + copied + new, st.total)
    shared_r, copied_r = shared[r], copied[r]
    has_source = place < shared_r + copied_r
    old = torch.where(has_source, st.table[torch.where(has_source, src[r] + place, 0)].long(), NONE)
    number = (torch.cumsum(copied + new, 0) - copied - new)[r] + place - shared_r      # among the fresh blocks
    fresh = free[number.clamp(0, st.blocks)]
    fresh = torch.where(has_source & (old < 0), NONE, fresh)
    entry = torch.where(place < shared_r, old, fresh)
    st.table[dst[r] + place] = entry.int()
    st.uses.index_add_(0, entry.clamp(min=0), (entry >= 0).int())
    is_copy = has_source & (place >= shared_r)
    at = (torch.cumsum(copied, 0) - copied)[r] + place - shared_r
    pairs = torch.full((st.max_pairs + 1, 2), NONE, dtype=torch.int32, device=DEV)
    pairs[torch.where(is_copy, at, st.max_pairs)] = torch.where((entry >= 0).unsqueeze(1), torch.stack([old, entry], 1), NONE).int()
    pairs[st.max_pairs] = NONE
    st.pairs.copy_(pairs[:st.max_pairs])
    st.totals.copy_(copied.sum().view(1))


def _free_plain(st):
    off, count = st.records.long().unbind(1)
    r, place = _entries(count, st.total)
    at = off[r] + place
    ids = st.table[at].long()
    st.uses.index_add_(0, ids.clamp(min=0), -(ids >= 0).int())
    st.table[at] = NONE


def _compact_plain(st):
    used = st.uses > 0
    ids = torch.arange(st.blocks, device=DEV)
    n_used = used.sum()
    holes, _, _ = _listed_places(~used & (ids < n_used))
    mover = used & (ids >= n_used)
    rank, n = _ranked(mover.flip(0))                   # the last block first
    rank = rank.flip(0)
    to = torch.where(mover, holes[rank], ids)
    pairs = torch.full((st.blocks + 1, 2), NONE, dtype=torch.int32, device=DEV)
    pairs[rank] = torch.stack([ids, to], 1).int()
    place = torch.arange(st.max_pairs, device=DEV).unsqueeze(1)
    st.pairs.copy_(torch.where(place < n, pairs[:st.max_pairs], NONE))
    moved = torch.zeros(st.blocks + 1, dtype=torch.int32, device=DEV)
    moved[torch.where(used, to, st.blocks)] = st.uses
    st.uses.copy_(moved[:st.blocks])
    named = st.table.long()
    st.table.copy_(torch.where(named >= 0, to[named.clamp(min=0)], named))
    st.totals.copy_(torch.stack([n, n_used]))


def _copy_plain(st):
    src, dst = st.pairs.long().unbind(1)
    for plane, scales in zip(st.planes, st.scales):
        x = plane.view(torch.int16 if scales is None else torch.uint8)
        x[dst] = x[src]
        if scales is not None:
            scales[dst] = scales[src]


PLAIN = {"sinks": _sinks_plain, "fork": _fork_plain, "free": _free_plain, "compact": _compact_plain, "copy": _copy_plain}


def run(state):
    if state.case["op"] in ("fork", "free", "compact"):
        state.live.copy_(state.saved)
    if own:
        return _own(state)
    PLAIN[state.case["op"]](state)
    return _result(state)


# ---- the same from the definitions: attention sequence by sequence in 64 bits, tables entry by entry on the host

def _exact_sinks(st):
    c = st.case
    T, h, hq, d = c["T"], c["h"], c["hq"], c["d"]
    out = torch.zeros(st.rows, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st.rows, hq, dtype=torch.float64, device=DEV)
    for row0, new, held, off in st.seqs.tolist():
        j = torch.arange(held, device=DEV)
        j = j[(j < c["sinks"]) | (j > held - new - c["window"])]
        ids = st.table[off + j // T].long()
        for head in range(h):
            kv = []
            for plane, scales in zip(st.planes, st.scales):
                x = (plane[ids, head, j % T] if c["hnd"] else plane[ids, j % T, head]).double()     # [keys, d]
                kv.append(x if scales is None else x * scales[ids, head].double().unsqueeze(1))
            group = slice(head * (hq // h), (head + 1) * (hq // h))
            step = max(1, (1 << 26) // (j.numel() * (hq // h)))
            for lo in range(0, new, step):
                hi = min(new, lo + step)
                q = st.q[row0 + lo:row0 + hi, group].double()                            # [rows, group, d]
                s = torch.tensordot(q, kv[0], dims=([2], [1])) / math.sqrt(d)
                p = torch.arange(held - new + lo, held - new + hi, device=DEV).unsqueeze(1)
                hidden = (j > p) | ((j <= p - c["window"]) & (j >= c["sinks"]))
                s = s.masked_fill(hidden.unsqueeze(1), -math.inf)
                z = torch.logsumexp(s, 2)
                lse[row0 + lo:row0 + hi, group] = z
                out[row0 + lo:row0 + hi, group] = torch.tensordot((s - z.unsqueeze(2)).exp(), kv[1], dims=1)
    return {"out": out, "lse": lse}


def _exact_table(st):
    c = st.case
    saved = st.saved.cpu().numpy()
    uses, table = [int(u) for u in saved[:st.blocks]], [int(t) for t in saved[st.blocks:]]
    if c["op"] == "free":
        for off, count in st.records.tolist():
            for e in range(off, off + count):
                if table[e] >= 0:
                    uses[table[e]] -= 1
                table[e] = NONE
        return {"uses": torch.tensor(uses, dtype=torch.int32), "table": torch.tensor(table, dtype=torch.int32)}
    pairs = []
    if c["op"] == "fork":
        free = iter([b for b, u in enumerate(uses) if u == 0])
        for src, dst, shared, copied, new in (r[:5] for r in st.records.tolist()):
            for e in range(shared + copied + new):
                old = table[src + e] if e < shared + copied else None
                block = old if e < shared else next(free, NONE)
                table[dst + e] = block
                if block >= 0:
                    uses[block] += 1
                if shared <= e < shared + copied:
                    pairs.append((old, block) if block >= 0 else (NONE, NONE))
        totals = [len(pairs)]
    else:
        n = sum(u > 0 for u in uses)
        holes = [b for b in range(n) if uses[b] == 0]
        movers = [b for b in range(st.blocks - 1, n - 1, -1) if uses[b] > 0]
        pairs = list(zip(movers, holes))
        to = dict(pairs)
        for a, b in pairs:
            uses[a], uses[b] = 0, uses[a]
        table = [to.get(t, t) for t in table]
        totals = [len(pairs), n]
    pairs += [(NONE, NONE)] * (st.max_pairs - len(pairs))
    return {"uses": torch.tensor(uses, dtype=torch.int32), "table": torch.tensor(table, dtype=torch.int32),
            "pairs": torch.tensor(pairs, dtype=torch.int32), "totals": torch.tensor(totals, dtype=torch.int32)}


def _exact_copy(st):
    got = {}
    for name, plane, scales in zip("kv", st.planes, st.scales):
        x = plane.double()
        for a, b in st.pairs.tolist():
            x[b].copy_(x[a])
        got[name] = x
        if scales is not None:
            y = scales.double()
            for a, b in st.pairs.tolist():
                y[b].copy_(y[a])
            got[name + "_scale"] = y
    return got


def exact(case, seed):
    st = prepare(case, seed)
    return {"sinks": _exact_sinks, "copy": _exact_copy}.get(case["op"], _exact_table)(st)


def work(case):
    """Each input that the operator has to read once, each output once; products over the keys that a query sees."""
    if case["op"] == "sinks":
        h, hq, d = case["h"], case["hq"], case["d"]
        new, held = _sequences(case)
        rows, e = int(new.sum()), 1 if case["cache"] == "e4m3" else 2
        first = _first_key(case, new, held)
        sinks = np.minimum(case["sinks"], first)
        scales = 8 * h * int((-(-held // case["T"]) - first // case["T"] + -(-sinks // case["T"])).sum()) if e == 1 else 0
        seen = 0
        for a, b in zip(new, held):
            place = np.arange(b - a, b)
            seen += int((np.minimum(place + 1, case["window"]) + np.minimum(case["sinks"], np.maximum(0, place + 1 - case["window"]))).sum())
        moved = 2 * e * h * d * int((held - first + sinks).sum()) + scales + 2 * 2 * rows * hq * d + 4 * rows * hq
        return {"bytes": moved, "flops": 4 * seen * hq * d}
    if case["op"] == "copy":
        e = 1 if case["cache"] == "e4m3" else 2
        block = case["T"] * case["h"] * case["d"] * e + (4 * case["h"] if e == 1 else 0)
        return {"bytes": case["pairs"] * (4 * block + 8), "flops": 0}
    n, _ = _rows_of(case)
    if case["op"] == "fork":       # which blocks are free; entries read and written, counts read and written, pairs
        _, shared, copied, new = _records(case)
        return {"bytes": 4 * case["blocks"] + int((16 * shared + 24 * copied + 12 * new).sum()) + 32 * n.size, "flops": 0}
    if case["op"] == "free":
        entries = int(n.sum()) if case["beams"] > 1 else n.size
        return {"bytes": 16 * entries + 8 * n.size, "flops": 0}
    # which blocks are in use; the entries of the tables read and written (counts and pairs of those that move come on top)
    return {"bytes": 4 * case["blocks"] + 8 * n.size * (int(n.max()) + 1), "flops": 0}
