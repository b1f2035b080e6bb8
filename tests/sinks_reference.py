"""Attention over the last tokens of a window and the first ones of a sequence, from its definition, in 64 bits on the CPU; and the error
that the operator's stated roundings allow.  Test infrastructure only."""
import math

import numpy as np

from kv_reference import E4M3, F32, UNIT


def attend(cache, dtype, seqs, table, q, group, sm_scale, window, sinks, table_len=None):
    """As kv_reference.attend, causal, and with its bounds (the arithmetic is the same: scores, weights, sums over the keys that are seen,
    the result), for queries that see key j of the keys up to their place if j > place - window, or j < sinks, or there is no window.
    A block is asked for if some query of the sequence sees a key of it."""
    T, d = cache.T, cache.d
    table_len = len(table) if table_len is None else table_len
    rows, hq = q.shape[:2]
    out, lse = np.full((rows, hq, d), np.nan), np.full((rows, hq), np.nan)
    out_err, lse_err = np.zeros((rows, hq, d)), np.zeros((rows, hq))
    u_w, status = UNIT["fp16" if cache.kind == "e4m3" else dtype], 0
    for row0, n_new, n_held, off in seqs:
        begin, j = n_held - n_new, np.arange(n_held)
        places = begin + np.arange(n_new)[:, None]
        visible = (j <= places) & ((j > places - window) | (j < sinks) | (window == 0))       # [queries, keys]
        there = np.zeros(n_held, bool)
        K, V = np.zeros((n_held, cache.h, d)), np.zeros((n_held, cache.h, d))
        for n in range(-(-n_held // T)):
            lo, hi, at = n * T, min(n_held, n * T + T), off + n
            if not visible[:, lo:hi].any():
                continue
            if at >= table_len or table[at] >= cache.blocks:
                status |= 1
                continue
            block = int(table[at])
            there[lo:hi] = True
            for x, plane, scales in zip((K, V), cache.planes, cache.scales):
                p = plane[block, :hi - lo]
                x[lo:hi] = E4M3[p] * scales[block].astype(np.float64)[None, :, None] if cache.kind == "e4m3" else p
        for i in range(n_new):
            seen = visible[i] & there
            for head in range(hq):
                kk, vv = K[seen, head // group], V[seen, head // group]
                if not seen.any():
                    out[row0 + i, head], lse[row0 + i, head] = 0.0, -math.inf
                    continue
                x = q[row0 + i, head].astype(np.float64)
                s = sm_scale * (kk @ x)
                top = s.max()
                w = np.exp(s - top)
                total = w.sum()
                w /= total
                with np.errstate(invalid="ignore"):
                    out[row0 + i, head], lse[row0 + i, head] = w @ vv, top + math.log(total)
                    size = abs(sm_scale) * (np.abs(kk) @ np.abs(x)).max()
                    ds = (d + 8) * F32 * size + 2 * F32 * np.abs(s).max() + 2.0 ** -21
                    sums = (len(w) / 8 + 64) * F32
                    mag = w @ np.abs(vv)
                    out_err[row0 + i, head] = (u_w + 2 * ds + 2 * sums) * mag * 1.01 + UNIT[dtype] * np.abs(w @ vv) * 1.01 + 2.0 ** -25
                lse_err[row0 + i, head] = ds + sums + 2 * F32 * abs(lse[row0 + i, head]) + 2.0 ** -22
    return out, lse, out_err, lse_err, status
