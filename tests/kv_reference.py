"""Appending to a paged cache and attention over it, from their definitions, in 64 bits on the CPU, sequence by sequence and
token by token; and the error that the operators' stated roundings allow.  Test infrastructure only."""
import math

import numpy as np
import torch

TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # largest relative error of one rounding to nearest
F32 = 2.0 ** -24


def e4m3_values():
    """The value of every code: 1 sign bit, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for code in range(256):
        e, m = code >> 3 & 15, code & 7
        x = m * 2.0 ** -9 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        v[code] = math.nan if code & 0x7f == 0x7f else -x if code & 0x80 else x
    return v


E4M3 = e4m3_values()
_POSITIVE = E4M3[:127]                              # ascending; code = index


def to_e4m3(x):
    """Codes of x (64 bits, an array): nearest, ties to the even code; beyond the largest value, the largest; NaN 0x7f or 0xff."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(x), 448.0)
    up = np.clip(np.searchsorted(_POSITIVE, a), 0, 126)
    down = np.maximum(up - 1, 0)
    gap_up, gap_down = _POSITIVE[up] - a, a - _POSITIVE[down]
    code = np.where((gap_up < gap_down) | ((gap_up == gap_down) & (up % 2 == 0)), up, down)
    code = np.where(np.isnan(x), 0x7f, code)
    return (code | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def scale_for(values):
    """Smallest power of two, at least 2^-64, with |x| <= 448 * it for all finite x."""
    v = np.abs(np.asarray(values, np.float64).ravel())
    top = float(v[np.isfinite(v)].max(initial=0.0))
    s = 2.0 ** -64
    while top > 448.0 * s:
        s *= 2.0
    return s


def rotate(x, cos, sin, interleaved):
    """x [..., d] (32-bit floats) by angles cos, sin [half]: each product and each sum rounded to 32 bits.  A copy."""
    x = np.array(x, np.float32)
    half = cos.size
    a = x[..., 0:2 * half:2].copy() if interleaved else x[..., :half].copy()
    b = x[..., 1:2 * half:2].copy() if interleaved else x[..., half:2 * half].copy()
    with np.errstate(all="ignore"):
        ra, rb = a * cos - b * sin, b * cos + a * sin
    if interleaved:
        x[..., 0:2 * half:2], x[..., 1:2 * half:2] = ra, rb
    else:
        x[..., :half], x[..., half:2 * half] = ra, rb
    return x


class Cache:
    """A pool on the CPU: planes [blocks, T, heads, d] as 32-bit values of a 16-bit type, or codes with scales [blocks, heads]."""

    def __init__(self, blocks, T, h, d, kind):
        self.T, self.h, self.d, self.kind, self.blocks = T, h, d, kind, blocks
        shape = (blocks, T, h, d)
        self.planes = [np.zeros(shape, np.uint8) if kind == "e4m3" else np.zeros(shape, np.float32) for _ in range(2)]
        self.scales = [np.ones((blocks, h), np.float32) for _ in range(2)]


def round16(x, kind):
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).to(TYPES[kind]).float().numpy()


def append(cache, dtype, seqs, table, q, k, v, rope, table_len=None):
    """seqs: (row0, n_new, n_held, table_off); q, k, v: [rows, heads, d] 32-bit floats.  rope: None or a dict of cos_sin, rot,
    interleaved, and pos [axes, rows] with pairs, or None.  Changes the cache; returns q_out (NaN where not written) and the
    status bits."""
    T, status = cache.T, 0
    table_len = len(table) if table_len is None else table_len
    q_out = np.full(q.shape, np.nan, np.float32)

    def turned(x, row, place):
        """x [heads, d] of a token, or None."""
        if rope is None:
            return np.array(x, np.float32)
        half = rope["rot"] // 2
        pairs = rope["pairs"] if rope["pos"] is not None else [half]
        pos = [int(p[row]) for p in rope["pos"]] if rope["pos"] is not None else [place]
        axis = [a for a, n in enumerate(pairs) for _ in range(n)]
        if any(pos[a] >= rope["cos_sin"].shape[0] for a in set(axis)):
            return None
        cs = rope["cos_sin"]
        cos = np.array([cs[pos[axis[j]], j] for j in range(half)], np.float32)
        sin = np.array([cs[pos[axis[j]], half + j] for j in range(half)], np.float32)
        return rotate(x, cos, sin, rope["interleaved"])

    for row0, n_new, n_held, off in seqs:
        begin = n_held - n_new
        fresh = {}                       # block number -> [(slot, row, k, v)]
        for i in range(n_new):
            row, place = row0 + i, begin + i
            kr = turned(k[row], row, place)
            if kr is None:
                status |= 32
                fresh.setdefault(place // T, [])
                continue
            q_out[row] = round16(turned(q[row], row, place), dtype)
            fresh.setdefault(place // T, []).append((place % T, row, kr, np.array(v[row], np.float32)))
        for n, tokens in fresh.items():
            at = off + n
            if at >= table_len or table[at] >= cache.blocks:
                status |= 1
                continue
            block = int(table[at])
            old = max(0, min(T, begin - n * T))      # slots of older tokens
            for plane, scales, which in zip(cache.planes, cache.scales, (2, 3)):
                if cache.kind != "e4m3":
                    for t in tokens:
                        plane[block, t[0]] = round16(t[which], cache.kind)
                    continue
                for head in range(cache.h):
                    s = scale_for([t[which][head] for t in tokens])
                    if old and scales[block, head] >= s:
                        s = float(scales[block, head])
                    elif old:
                        was = E4M3[plane[block, :old, head]] * float(scales[block, head])
                        plane[block, :old, head] = to_e4m3(was / s)
                    for t in tokens:
                        plane[block, t[0], head] = to_e4m3(t[which][head].astype(np.float64) / s)
                    scales[block, head] = s
    return q_out, status


def attend(cache, dtype, seqs, table, q, group, sm_scale, causal=True, window=0, table_len=None):
    """out, lse in 64 bits, and for each value of out and lse how far the operator may be from it:

    a score: the sum of d products in 32 bits, any order, then two products and (e4m3) a sum: |error| <= (d + 8) 2^-24 sum|q k|
    |scale|, taken with the largest over the keys, and 2^-23 of the scores' size (base-2 logarithms, differences);
    a weight: one rounding to the type that meets the values; exp2, log2 and reciprocals to 2^-21 in all;
    sums of weights and of products, in 32 bits over L keys in tiles, split and joined: (L/8 + 64) 2^-24 of the sum of magnitudes;
    the result: one rounding to dtype (and 2^-25 for fp16's smallest steps)."""
    T, d = cache.T, cache.d
    table_len = len(table) if table_len is None else table_len
    rows, hq = q.shape[:2]
    out, lse = np.full((rows, hq, d), np.nan), np.full((rows, hq), np.nan)
    out_err, lse_err = np.zeros((rows, hq, d)), np.zeros((rows, hq))
    u_w, status = UNIT["fp16" if cache.kind == "e4m3" else dtype], 0
    for row0, n_new, n_held, off in seqs:
        begin = n_held - n_new
        there = np.zeros(n_held, bool)
        K, V = np.zeros((n_held, cache.h, d)), np.zeros((n_held, cache.h, d))
        low = max(0, begin + 1 - window) if window else 0
        for n in range(-(-n_held // T)):
            lo, hi = n * T, min(n_held, n * T + T)
            at = off + n
            if at >= table_len or table[at] >= cache.blocks:
                status |= 1 if hi > low else 0
                continue
            block = int(table[at])
            there[lo:hi] = True
            for x, plane, scales in zip((K, V), cache.planes, cache.scales):
                p = plane[block, :hi - lo]
                x[lo:hi] = E4M3[p] * scales[block].astype(np.float64)[None, :, None] if cache.kind == "e4m3" else p
        j = np.arange(n_held)
        for i in range(n_new):
            seen = there & (j <= begin + i) if causal else there.copy()
            if window:
                seen &= j > begin + i - window
            for head in range(hq):
                kk, vv = K[seen, head // group], V[seen, head // group]
                if not seen.any():
                    out[row0 + i, head], lse[row0 + i, head] = 0.0, -math.inf
                    continue
                x = q[row0 + i, head].astype(np.float64)
                s = sm_scale * (kk @ x)
                top = s.max()
                w = np.exp(s - top)
                l = w.sum()
                w /= l
                out[row0 + i, head], lse[row0 + i, head] = w @ vv, top + math.log(l)
                size = abs(sm_scale) * (np.abs(kk) @ np.abs(x)).max()
                ds = (d + 8) * F32 * size + 2 * F32 * np.abs(s).max() + 2.0 ** -21
                sums = (len(w) / 8 + 64) * F32
                mag = w @ np.abs(vv)
                out_err[row0 + i, head] = (u_w + 2 * ds + 2 * sums) * mag * 1.01 + UNIT[dtype] * np.abs(w @ vv) * 1.01 + 2.0 ** -25
                lse_err[row0 + i, head] = ds + sums + 2 * F32 * abs(lse[row0 + i, head]) + 2.0 ** -22
    return out, lse, out_err, lse_err, status
