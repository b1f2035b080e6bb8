"""Timed cases of the operators that fill a paged KV cache and read it: appending and attention.

  append   tutti_kv_append: new tokens' queries and keys are rotated by their positions (one axis, or time / height /
           width), keys and values go to their places in the paged pool.  A pool of 8-bit elements holds e4m3 values
           with one scale, a power of two, for each block and head: a block whose largest magnitude grows is rescaled.
  attend   tutti_kv_attend: attention of the new tokens' queries over everything their sequences hold in the pool,
           causal, with an optional sliding window, over 16-bit blocks or e4m3 blocks with their scales.

`own` chooses between the plain form in elementary torch operations and the framework's calls.  A case says what one layer
of a serving step looks like: how many sequences, how many tokens each has brought along and holds in all.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
FLOOR = -64                  # exponent of the smallest scale of an 8-bit block
LARGEST = 448.0              # largest e4m3 value
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}

# T: tokens a block; h: KV heads; hq: query heads; d: head size; cache: type of the pool; x: type of queries, keys, values
BASE = dict(op="attend", T=16, h=8, hq=32, d=128, x="bf16", cache="bf16", hnd=False, seqs=1, new=1, new_spread=False,
            held=1024, held_spread="even", window=0, rot=128, axes=1, interleaved=False)


def _case(name, **kw):
    return dict(BASE, name=name, **kw)


def listed():
    return [
        # one running sequence decodes: its token's key and value go to the cache; the smallest call
        _case("append_one", op="append", held=4099),
        # a decode step of 256 running sequences, 8-bit cache: some blocks are just begun, most are open ones
        _case("append_decode_256_e4m3", op="append", cache="e4m3", seqs=256, new=256, held=1200, held_spread="zipf"),
        # chunks of prompts, 8,191 tokens in 7 sequences, that go on in the middle of a block, 8-bit cache
        _case("append_prompts_8k_e4m3", op="append", cache="e4m3", seqs=7, new=8191, new_spread=True, held=3000,
              held_spread="zipf"),
        # images and video in a prompt: 16,384 tokens with positions in time, height and width, head-major pool
        _case("append_video_16k", op="append", hnd=True, seqs=4, new=16384, new_spread=True, held=500, axes=3),
        # a one-layer model of 2 heads x 64 and its 512-token prefix: latency
        _case("decode_tiny", T=16, h=2, hq=4, d=64, x="fp16", cache="fp16", held=512, rot=64),
        # 8B shape, one sequence with a restored 32K-token prefix, 16-bit cache (128 MiB)
        _case("decode_one_32k", held=32768),
        # 70B shape, one sequence of 128K tokens, 8-bit cache (256 MiB)
        _case("decode_one_128k_e4m3", hq=64, held=131072, cache="e4m3"),
        # a serving batch: 64 sequences of Zipf-distributed lengths, 8-bit cache
        _case("decode_batch64_e4m3", seqs=64, new=64, held=6000, held_spread="zipf", cache="e4m3"),
        # drafts verified: 32 sequences bring 5 tokens each, as one rank of a tensor-parallel group of 8 holds them
        _case("verify_32x5_tp8", T=32, h=1, hq=8, seqs=32, new=160, held=8000, held_spread="zipf"),
        # a chunk of a long prompt: 2,048 tokens behind 30,000 that are there, 8-bit cache
        _case("chunk_2k_behind_30k_e4m3", new=2048, held=32048, cache="e4m3"),
        # prompts of uneven lengths, 8,001 tokens in 5 sequences, nothing before them
        _case("prompts_8k", seqs=5, new=8001, new_spread=True, held=0),
        # 5 heads x 80, sliding window: a prompt's chunk and decoding sequences in one step, head-major 8-bit pool
        _case("mixed_window_5x80_e4m3", h=5, hq=20, d=80, rot=80, x="fp16", cache="e4m3", hnd=True, T=32, seqs=12, new=1511,
              new_spread="one", held=7000, held_spread="zipf", window=4096),
    ]


def _log(rng, lo, hi):
    """A whole number between lo and hi, uniform over its logarithm."""
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(("append", "attend", "attend"))
    while True:
        h, group = rng.choice((1, 2, 4, 5, 8, 8)), rng.choice((1, 2, 4, 4, 5, 8))
        d = rng.choice((64, 80, 96, 112, 128, 128, 128))
        if h * group <= 64:
            break
    x = rng.choice(("bf16", "bf16", "fp16"))
    case = dict(BASE, op=op, T=rng.choice((16, 16, 32, 64)), h=h, hq=h * group, d=d, rot=rng.choice((d, d, d // 2)), x=x,
                cache=rng.choice((x, "e4m3")), hnd=rng.random() < 0.3, interleaved=rng.random() < 0.3,
                axes=rng.choice((1, 1, 3)), held_spread=rng.choice(("even", "zipf")))
    if op == "append":
        new = _log(rng, 1, 16384)
        case.update(new=new, seqs=min(new, _log(rng, 1, 256)), new_spread=rng.random() < 0.5, held=_log(rng, 1, 6000))
        return case
    case["window"] = rng.choice((0, 0, 0, _log(rng, 128, 4096)))
    kind = rng.choice(("decode", "decode", "verify", "prompt", "mixed"))
    if kind in ("decode", "verify"):
        seqs = _log(rng, 1, 128)
        each = 1 if kind == "decode" else rng.randint(2, 8)
        held = _log(rng, 64, max(65, min(131072, 3000000 // (seqs * h))))
        case.update(seqs=seqs, new=seqs * each, held=max(held, each))
    else:
        seqs = _log(rng, 1, 8) if kind == "prompt" else rng.randint(3, 12)
        new = max(seqs, _log(rng, 64, 4096))
        most = 1200000000 // (h * group * new * (seqs if kind == "mixed" else 1))     # scores of the plain form
        held = 0 if rng.random() < 0.3 else _log(rng, 64, max(65, min(30000, most)))
        case.update(seqs=seqs, new=new, new_spread=True if kind == "prompt" else "one", held=held)
    return case


# ---- what a case's sequences look like: the same for every seed (they decide the outputs' sizes)

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
    rng = np.random.default_rng(20260503)
    new = _shares(case["new"], n, case["new_spread"], rng)
    if case["held_spread"] == "zipf":     # lengths over 64 ranks, as a mix of long and short contexts has them
        ranks = np.arange(1, 65, dtype=np.float64)
        p = ranks ** -1.1
        w = rng.choice(ranks, size=n, p=p / p.sum()) * rng.uniform(0.3, 1.0, size=n)
        held = np.floor(case["held"] * np.minimum(w / w.mean(), 5.0)).astype(np.int64)
    else:
        held = np.full(n, case["held"], np.int64) - np.arange(n) % 7 * (1 if n > 1 else 0)
    if case["op"] == "append":
        return new, np.maximum(held, 0) + new
    return new, np.maximum(held, new) if case["held"] else new


class _State:
    pass


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


def prepare(case, seed):
    rng = np.random.default_rng([seed, case["new"], case["held"]])
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    T, h, hq, d, n = case["T"], case["h"], case["hq"], case["d"], case["seqs"]
    new, held = _sequences(case)
    rows, need = int(new.sum()), -(-held // T)
    blocks = int(need.sum()) + int(need.sum()) // 8 + 3
    st = _State()
    st.case, st.rows, st.blocks = case, rows, blocks
    st.max_new, st.max_held = int(new.max()), int(held.max())
    table = rng.permutation(blocks)[:int(need.sum())].astype(np.int32)
    row0, off = np.cumsum(new) - new, np.cumsum(need) - need
    seqs = np.stack([row0, new, held, off], 1).astype(np.int32)
    st.table, st.seqs = torch.from_numpy(table).to(DEV), torch.from_numpy(seqs).to(DEV)
    first = (held - new) // T
    st.touched = int((-(-held // T) - first).sum())   # blocks that get a new token

    # the pool: what earlier tokens left there, blocks of uneven magnitude, a few large channels in the keys
    x = TYPES[case["x"]]
    st.k_scale = st.v_scale = None
    st.planes = []
    for kind in range(2):
        plane = torch.empty(_plane(case, blocks), dtype=TYPES[case["cache"]], device=DEV)
        scales = torch.empty(blocks, -(-h // 4) * 4, device=DEV)
        loud = torch.ones(d, device=DEV)
        if kind == 0:
            loud[torch.randint(0, d, (3,), generator=gen, device=DEV)] = 4.0
        step = max(1, (1 << 27) // (T * h * d))
        for lo in range(0, blocks, step):
            hi = min(blocks, lo + step)
            v = torch.randn(_plane(case, hi - lo), generator=gen, device=DEV) * loud
            v *= torch.exp(0.3 * torch.randn(hi - lo, 1, 1, 1, generator=gen, device=DEV))
            if case["cache"] == "e4m3":
                plane[lo:hi], scales[lo:hi] = _quantised(v, 2 if case["hnd"] else 1, scales.shape[1])
            else:
                plane[lo:hi] = v.to(x)
        st.planes.append(plane)
        if case["cache"] == "e4m3":
            if kind == 0:
                st.k_scale = scales
            else:
                st.v_scale = scales
    # one projection gives queries, keys and values side by side, as a fused product leaves them
    st.qkv = torch.randn(rows, hq + 2 * h, d, generator=gen, device=DEV).to(x)
    st.q, st.k, st.v = st.qkv[:, :hq], st.qkv[:, hq:hq + h], st.qkv[:, hq + h:]
    if case["op"] == "append":
        st.q_out = torch.empty(rows, hq, d, dtype=x, device=DEV)
        # angles: cosines, then sines, for each position
        half = case["rot"] // 2
        pairs = [half] if case["axes"] == 1 else [half - 2 * (3 * half // 8), 3 * half // 8, 3 * half // 8]
        positions = st.max_held if case["axes"] == 1 else max(st.max_held, 512)
        angle = torch.arange(positions, device=DEV, dtype=torch.float64).unsqueeze(1)
        angle = angle * 10000.0 ** (-torch.arange(half, device=DEV, dtype=torch.float64) / half)
        st.cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float()
        st.pairs, st.pos = pairs, None
        if case["axes"] > 1:       # places in a video: frames of 16 x 24 patches
            place = torch.from_numpy(np.concatenate([np.arange(a, b) for a, b in zip(held - new, held)])).to(DEV)
            st.pos = torch.stack([place // 384, place // 24 % 16, place % 24]).to(torch.int32)
    else:
        st.out = torch.empty(rows, hq, d, dtype=x, device=DEV)
        st.lse = torch.empty(rows, hq, device=DEV)
    st.handles = None
    return st


# ---- the framework's calls

def _handles(st):
    """What a program makes once for a step and uses in every layer: the pool's and the batch's records, work memory."""
    from paper_2605_03375_amd import binding as B
    c = st.case
    h = _State()
    h.B = B
    h.pool = B.make_pool(st.planes[0], st.planes[1], num_blocks=st.blocks, block_tokens=c["T"], num_kv_heads=c["h"],
                         head_dim=c["d"], elt_bytes=st.planes[0].element_size(),
                         pool_layout=B.LAYOUT_HND if c["hnd"] else B.LAYOUT_NHD)
    h.scales = None if st.k_scale is None else B.make_scales(st.k_scale, st.v_scale)
    h.batch = B.make_batch(st.seqs, c["seqs"], st.max_new, st.table, st.table.numel(), st.rows)
    h.dtype = {"bf16": B.BF16, "fp16": B.FP16}[c["x"]]
    if c["op"] == "append":
        h.rope = B.make_rope(st.cos_sin, c["rot"], d_pos=st.pos, pairs=st.pairs, interleaved=c["interleaved"])
        h.rows = [B.make_rows(t) for t in (st.q, st.q_out, st.k, st.v)]
        h.result = {"q": st.q_out, "k": st.planes[0], "v": st.planes[1]}
        if st.k_scale is not None:
            h.result.update(k_scale=st.k_scale, v_scale=st.v_scale)
    else:
        h.attn = B.make_attn(c["hq"], h.dtype, 1.0 / math.sqrt(c["d"]), causal=True, window=c["window"])
        h.rows = [B.make_rows(t) for t in (st.q, st.out)]
        h.work = torch.empty(B.tutti_kv_attend_work_bytes(h.pool, h.batch, h.attn), dtype=torch.uint8, device=DEV)
        h.result = {"out": st.out, "lse": st.lse}
    return h


def _own(st):
    if st.handles is None:
        st.handles = _handles(st)
    h = st.handles
    if st.case["op"] == "append":
        h.B.tutti_kv_append(h.pool, h.scales, h.batch, h.rope, *h.rows, st.case["hq"], h.dtype)
    else:
        h.B.tutti_kv_attend(h.pool, h.scales, h.batch, h.attn, *h.rows, st.lse, h.work, h.work.numel())
    return h.result


# ---- the plain form

def _owners(st):
    """For each row: its sequence, and its place in it."""
    row0, new, held, off = st.seqs.long().unbind(1)
    row = torch.arange(st.rows, device=DEV)
    s = torch.searchsorted(row0 + new, row, right=True)
    return s, held[s] - new[s] + row - row0[s]


def _rotated(st, x, place):
    """x [rows, heads, d] with its first `rot` values rotated, in 32 bits."""
    c = st.case
    half = c["rot"] // 2
    if c["axes"] == 1:
        cos, sin = st.cos_sin[place].unsqueeze(1).split(half, 2)
    else:
        axis = torch.repeat_interleave(torch.arange(3, device=DEV), torch.tensor(st.pairs, device=DEV), output_size=half)
        pos, j = st.pos.long()[axis].T, torch.arange(half, device=DEV)        # [rows, half]
        cos, sin = st.cos_sin[pos, j].unsqueeze(1), st.cos_sin[pos, j + half].unsqueeze(1)
    x = x.float()
    r, rest = x[..., :c["rot"]], x[..., c["rot"]:]
    a, b = (r[..., 0::2], r[..., 1::2]) if c["interleaved"] else (r[..., :half], r[..., half:])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    r = torch.stack([ra, rb], 3).flatten(2) if c["interleaved"] else torch.cat([ra, rb], 2)
    return torch.cat([r, rest], 2)


def _append_plain(st):
    c = st.case
    T = c["T"]
    s, place = _owners(st)
    row0, new, held, off = st.seqs.long().unbind(1)
    st.q_out.copy_(_rotated(st, st.q, place))
    k, v = _rotated(st, st.k, place), st.v.float()
    block, slot = st.table.long()[off[s] + place // T], place % T
    result = {"q": st.q_out, "k": st.planes[0], "v": st.planes[1]}
    if c["cache"] != "e4m3":
        for plane, x in zip(st.planes, (k, v)):
            (plane.transpose(1, 2) if c["hnd"] else plane)[block, slot] = x.to(plane.dtype)
        return result
    # every block that gets a token: which of its slots are old ones, which new ones, and their rows
    begin = held - new
    count = (held - 1) // T - begin // T + 1
    u = torch.repeat_interleave(torch.arange(c["seqs"], device=DEV), count, output_size=st.touched)
    at = begin[u] // T + torch.arange(st.touched, device=DEV) - (torch.cumsum(count, 0) - count)[u]
    block = st.table.long()[off[u] + at]
    p = at.unsqueeze(1) * T + torch.arange(T, device=DEV)                      # [touched, T]
    is_old = (p < begin[u].unsqueeze(1)).unsqueeze(2).unsqueeze(3)
    is_new = ((p >= begin[u].unsqueeze(1)) & (p < held[u].unsqueeze(1))).unsqueeze(2).unsqueeze(3)
    row = (row0[u] - begin[u]).unsqueeze(1) + p
    row = row.clamp(0, st.rows - 1)
    for plane, scales, x in zip(st.planes, (st.k_scale, st.v_scale), (k, v)):
        tokens = plane.transpose(1, 2) if c["hnd"] else plane                  # [blocks, T, h, d]
        before = tokens.view(torch.uint8)[block]
        x = torch.where(is_new, x[row], 0.0)
        m, e = torch.frexp(x.abs().amax(dim=(1, 3)))
        scale = torch.ldexp(torch.ones_like(m), torch.clamp(e - 9 + (m > 0.875).int(), min=FLOOR))
        held_scale = scales[block, :c["h"]]
        scale = torch.where(is_old[:, 0, :, 0], torch.maximum(scale, held_scale), scale)
        old = before.view(plane.dtype).float() * held_scale.unsqueeze(1).unsqueeze(3)
        y = (torch.where(is_new, x, old) / scale.unsqueeze(1).unsqueeze(3)).to(torch.float8_e4m3fn)
        kept = torch.where(is_old | is_new, y.view(torch.uint8), before)
        tokens.view(torch.uint8)[block] = kept
        scales[block, :c["h"]] = scale
    result.update(k_scale=st.k_scale, v_scale=st.v_scale)
    return result


def _attend_plain(st):
    c = st.case
    T, h, hq, d, n = c["T"], c["h"], c["hq"], c["d"], c["seqs"]
    row0, new, held, off = st.seqs.long().unbind(1)
    j = torch.arange(st.max_held, device=DEV)
    there = j < held.unsqueeze(1)                                              # [n, keys]
    index = torch.where(there, off.unsqueeze(1) + j // T, 0)
    block, slot = st.table.long()[index], (j % T).expand(n, -1)
    keys, values = [], []
    for plane, scales, to in zip(st.planes, (st.k_scale, st.v_scale), (keys, values)):
        x = plane.view(torch.int16 if scales is None else torch.uint8)                # (indexed as they lie)
        x = (x.transpose(1, 2) if c["hnd"] else x)[block, slot].view(plane.dtype).float()       # [n, keys, h, d]
        if scales is not None:
            x *= scales[block][..., :h].unsqueeze(3)
        to.append(x.masked_fill_(~there.unsqueeze(2).unsqueeze(3), 0.0).transpose(1, 2).contiguous())
    i = torch.arange(st.max_new, device=DEV)
    q = st.q.float()[(row0.unsqueeze(1) + i).clamp(max=st.rows - 1)]           # [n, new, hq, d]
    q = q.transpose(1, 2).reshape(n, h, hq // h * st.max_new, d)
    scores = torch.matmul(q, keys.pop().transpose(2, 3)) * (1.0 / math.sqrt(d))
    scores = scores.view(n, h, hq // h, st.max_new, st.max_held)
    place = (held - new).unsqueeze(1) + i                                      # [n, new]
    seen = there.unsqueeze(1) & (j <= place.unsqueeze(2))
    if c["window"]:
        seen = seen & (j > place.unsqueeze(2) - c["window"])
    scores.masked_fill_(~seen.unsqueeze(1).unsqueeze(1), -math.inf)
    top = scores.amax(4, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    weights = scores.sub_(top).exp_()
    total = weights.sum(4, keepdim=True)
    out = torch.matmul(weights.view(n, h, -1, st.max_held), values.pop()).view(n, hq, st.max_new, d)
    out = out / total.view(n, hq, st.max_new, 1)
    lse = (top + total.log()).view(n, hq, st.max_new)
    s, at = _owners(st)
    i = at - (held - new)[s]
    st.out.copy_(out[s, :, i])
    st.lse.copy_(lse[s, :, i])
    return {"out": st.out, "lse": st.lse}


def run(state):
    if own:
        return _own(state)
    return _append_plain(state) if state.case["op"] == "append" else _attend_plain(state)


# ---- the same from the definitions, sequence by sequence, in 64 bits

def _to_e4m3(x):
    """x in 64 bits rounded to e4m3, ties to even: 3 bits behind the leading one, steps of 2^-9 below 2^-6."""
    m, e = torch.frexp(x)
    step = torch.ldexp(torch.ones_like(x), torch.clamp(e - 4, min=-9))
    return torch.clamp(torch.round(x / step) * step, -LARGEST, LARGEST)


def _exact_append(st):
    c = st.case
    T, half = c["T"], c["rot"] // 2
    axis = [a for a, k in enumerate(st.pairs) for _ in range(k)]
    planes = [p.double() for p in st.planes]
    scales = [None, None] if st.k_scale is None else [st.k_scale.double(), st.v_scale.double()]
    q_out = st.q.double().clone()
    k_all = st.k.double().clone()
    for row0, new, held, off in st.seqs.tolist():
        rows = slice(row0, row0 + new)
        place = torch.arange(held - new, held, device=DEV)
        for j in range(half):
            pos = place if st.pos is None else st.pos[axis[j], rows].long()
            cos, sin = st.cos_sin[pos, j].double().unsqueeze(1), st.cos_sin[pos, half + j].double().unsqueeze(1)
            a, b = (2 * j, 2 * j + 1) if c["interleaved"] else (j, j + half)
            for x in (q_out, k_all):
                u, w = x[rows, :, a].clone(), x[rows, :, b].clone()
                x[rows, :, a] = u * cos - w * sin
                x[rows, :, b] = u * sin + w * cos
        for plane, scale, x in zip(planes, scales, (k_all, st.v.double())):
            if c["cache"] != "e4m3":
                block, slot = st.table[off + place // T].long(), place % T
                if c["hnd"]:
                    plane[block, :, slot] = x[rows]
                else:
                    plane[block, slot] = x[rows]
                continue
            # whole sequence at once: its touched blocks, from the one that the first new token falls into
            first, last = (held - new) // T, (held - 1) // T
            ids = st.table[off + first:off + last + 1].long()
            body = torch.zeros((last + 1 - first) * T, c["h"], c["d"], dtype=torch.float64, device=DEV)
            at = held - new - first * T
            body[at:at + new] = x[rows]
            body = body.view(-1, T, c["h"], c["d"])
            need = body.abs().amax(dim=(1, 3))
            m, e = torch.frexp(need / LARGEST)          # smallest power of two that is no less
            power = torch.where(m == 0.5, e - 1, e)
            power = torch.where(need == 0, FLOOR, power).clamp(min=FLOOR)
            s = torch.ldexp(torch.ones_like(need), power)
            was = scale[ids, :c["h"]]
            tokens = (plane.transpose(1, 2) if c["hnd"] else plane)[ids]
            if at:
                s[0] = torch.maximum(s[0], was[0])
                body[0, :at] = tokens[0, :at] * was[0].unsqueeze(1)
            y = _to_e4m3(body / s.unsqueeze(1).unsqueeze(3)).flatten(0, 1)
            flat = tokens.flatten(0, 1).clone()
            flat[:at + new] = y[:at + new]
            flat = flat.view_as(tokens)
            plane[ids] = flat.transpose(1, 2) if c["hnd"] else flat
            scale[ids, :c["h"]] = s
    result = {"q": q_out, "k": planes[0], "v": planes[1]}
    if scales[0] is not None:
        result.update(k_scale=scales[0], v_scale=scales[1])
    return result


def _exact_attend(st):
    c = st.case
    T, h, hq, d = c["T"], c["h"], c["hq"], c["d"]
    out = torch.zeros(st.rows, hq, d, dtype=torch.float64, device=DEV)
    lse = torch.zeros(st.rows, hq, dtype=torch.float64, device=DEV)
    for row0, new, held, off in st.seqs.tolist():
        ids = st.table[off:off + -(-held // T)].long()
        for head in range(h):
            kv = []
            for plane, scales in zip(st.planes, (st.k_scale, st.v_scale)):
                x = (plane[ids, head] if c["hnd"] else plane[ids, :, head]).double()     # [blocks, T, d]
                if scales is not None:
                    x = x * scales[ids, head].double().view(-1, 1, 1)
                kv.append(x.flatten(0, 1)[:held])
            group = slice(head * (hq // h), (head + 1) * (hq // h))
            step = max(1, (1 << 26) // (held * (hq // h)))
            for lo in range(0, new, step):
                hi = min(new, lo + step)
                q = st.q[row0 + lo:row0 + hi, group].double()                            # [rows, group, d]
                s = torch.tensordot(q, kv[0], dims=([2], [1])) / math.sqrt(d)
                place = torch.arange(held - new + lo, held - new + hi, device=DEV).unsqueeze(1)
                j = torch.arange(held, device=DEV)
                hidden = j > place
                if c["window"]:
                    hidden = hidden | (j <= place - c["window"])
                s = s.masked_fill(hidden.unsqueeze(1), -math.inf)
                z = torch.logsumexp(s, 2)
                lse[row0 + lo:row0 + hi, group] = z
                out[row0 + lo:row0 + hi, group] = torch.tensordot((s - z.unsqueeze(2)).exp(), kv[1], dims=1)
    return {"out": out, "lse": lse}


def exact(case, seed):
    st = prepare(case, seed)
    return _exact_append(st) if case["op"] == "append" else _exact_attend(st)


def work(case):
    """Each input that the operator has to read once, each output once; products over the keys that a query sees."""
    h, hq, d = case["h"], case["hq"], case["d"]
    new, held = _sequences(case)
    rows, e = int(new.sum()), 1 if case["cache"] == "e4m3" else 2
    if case["op"] == "append":
        inputs = 2 * rows * (hq + 2 * h) * d
        outputs = 2 * rows * hq * d + e * rows * 2 * h * d
        if e == 1:
            outputs += 8 * h * int(((held - 1) // case["T"] - (held - new) // case["T"] + 1).sum())   # scales
        angles = 4 * rows * case["rot"]
        return {"bytes": inputs + outputs + angles, "flops": 3 * rows * (hq + h) * case["rot"]}
    window = case["window"] or 1 << 40
    first = np.maximum(0, held - new + 1 - window)                  # of the keys that any query sees
    scales = 8 * h * int((-(-held // case["T"]) - first // case["T"]).sum()) if e == 1 else 0
    seen = sum(int(np.minimum(np.arange(b - a + 1, b + 1), window).sum()) for a, b in zip(new, held))
    moved = 2 * e * h * d * int((held - first).sum()) + scales + 2 * 2 * rows * hq * d + 4 * rows * hq
    return {"bytes": moved, "flops": 4 * seen * hq * d}
