"""Attention whose parts are long, whose splits are many or whose sequences are more than 64: what the kernels look up again on their way,
and every shape of the join.  Against 64 bits on the GPU; sequences share their blocks, which attention only reads."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
from paper_2605_03375_amd import binding as B
from test_kv_ops import DEV, Step, run_attend, same

gpu = pytest.mark.gpu
SLOTS = 512          # workgroups that the plan takes to be on the device at once


def tiles(n):
    return -(-n // 32)


def units(st):
    """Row tiles of all sequences and (groups of) KV heads: as many workgroups, if nothing is split."""
    most = max(n_new for _, n_new, _, _ in st.seqs) * st.group
    rows = 16 if most <= 16 else 32 if most <= 32 else 128
    side = next((n for n in (4, 5, 3, 2) if st.h % n == 0), 1) if rows < 128 else 1
    return sum(-(-n_new * st.group // rows) for _, n_new, _, _ in st.seqs) * (st.h // side)


def of_one(seqs, **kw):
    """A step of sequences (new, held) over the blocks of one that is as long as the longest."""
    n_held = max(b for _, b in seqs)
    st = Step([(1, n_held)], **kw)
    rng = np.random.default_rng(7)
    row = np.concatenate([[0], np.cumsum([a for a, _ in seqs])])
    st.seqs, st.rows = [(int(r), a, b, 0) for r, (a, b) in zip(row, seqs)], int(row[-1])
    st.q, st.k, st.v = (ref.round16(rng.standard_normal((st.rows, n, st.d)), st.dtype) for n in (st.hq, st.h, st.h))
    return st


def check(st, window=0):
    """run_attend against 64 bits within the bound of kv_reference.attend."""
    out, lse, status = run_attend(st.to_gpu(), window=window)
    n_held, scale = max(s[2] for s in st.seqs), 1.0 / math.sqrt(st.d)
    places = np.arange(n_held)
    ids = st.table[places // st.T]
    there = ids < st.blocks
    kv = []
    for plane, scales in zip(st.cpu.planes, st.cpu.scales):
        x = plane[np.where(there, ids, 0), places % st.T]
        x = ref.E4M3[x] * scales[np.where(there, ids, 0)][:, :, None].astype(np.float64) if st.kind == "e4m3" else x
        kv.append(torch.from_numpy(np.where(there[:, None, None], x, 0.0)).double().to(DEV))
    q, j, d_there = torch.from_numpy(st.q).double().to(DEV), torch.arange(n_held, device=DEV), torch.from_numpy(there).to(DEV)
    unit, u_w = ref.UNIT[st.dtype], ref.UNIT["fp16" if st.kind == "e4m3" else st.dtype]
    d_out, d_lse = torch.from_numpy(out).double().to(DEV), torch.from_numpy(lse).double().to(DEV)
    want_status = 0
    for row0, n_new, held, _ in st.seqs:
        place = torch.arange(held - n_new, held, device=DEV).unsqueeze(1)
        seen = (j <= place) & d_there
        if window:
            seen = seen & (j > place - window)
        low = max(0, held - n_new + 1 - window) // st.T * st.T if window else 0
        want_status |= 0 if there[low:held].all() else B.ST_BAD_BLOCK
        rows = slice(row0, row0 + n_new)
        for head in range(st.h):
            group = slice(head * st.group, (head + 1) * st.group)
            k, v = kv[0][:, head].contiguous(), kv[1][:, head].contiguous()
            x = q[rows, group]
            s = (torch.tensordot(x, k, dims=([2], [1])) * scale).masked_fill(~seen.unsqueeze(1), -math.inf)
            z = torch.logsumexp(s, 2, keepdim=True)
            w = torch.where(z == -math.inf, 0.0, (s - z).exp())
            want, mag = torch.tensordot(w, v, dims=1), torch.tensordot(w, v.abs(), dims=1)
            size = scale * torch.tensordot(x.abs(), k.abs(), dims=([2], [1])).masked_fill(~seen.unsqueeze(1), 0.0).amax(2, keepdim=True)
            biggest = s.abs().masked_fill(~seen.unsqueeze(1), 0.0).amax(2, keepdim=True)
            n = seen.sum(1)[:, None, None].double()
            ds = (st.d + 8) * ref.F32 * size + 2 * ref.F32 * biggest + 2.0 ** -21
            sums = (n / 8 + 64) * ref.F32
            bound = (u_w + 2 * ds + 2 * sums) * mag * 1.01 + unit * want.abs() * 1.01 + 2.0 ** -25
            assert bool(((d_out[rows, group] - want).abs() <= bound).all()), (row0, head)
            z, got = z.squeeze(2), d_lse[rows, group]
            near = (got - z).abs() <= (ds + sums).squeeze(2) + 2 * ref.F32 * z.abs() + 2.0 ** -22
            assert bool((near | ((z == -math.inf) & (got == -math.inf))).all()), (row0, head)
    assert status == want_status
    for fill in (0x00, 0x7f):
        again = run_attend(st, window=window, work_fill=fill)
        assert same(out, again[0]) and same(lse, again[1])


def gone(st, *blocks):
    for b in blocks:
        st.table[b] = 0xffffffff


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("h,n_held,n_seq", [(4, 3001, 600), (1, 6007, 600), (2, 4100, 600)])
@pytest.mark.parametrize("window", [0, 2500])
def test_few_queries_of_whole_long_sequences(window, h, n_held, n_seq, T, cache):
    """More than 32 tiles of 32 keys for each wavefront (of one, four or two that share a head's): looked up again, with blocks that are not
    there on both sides of it; lengths that end anywhere in a tile."""
    st = of_one([(1, n_held - i % 70) for i in range(n_seq)], T=T, h=h, d=64, cache="e4m3" if cache == "e4m3" else None)
    waves = {4: 1, 1: 4, 2: 2}[h]
    assert units(st) >= SLOTS and tiles(min(n_held, window or n_held) - 70) > 32 * waves or window
    gone(st, 40, 1030 // T, 1025 // T + 1, 2200 // T, 2900 // T)
    check(st, window)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (80, "fp16"), (128, "bf16")])
@pytest.mark.parametrize("window", [0, 1500])
def test_many_queries_of_whole_long_sequences(window, d, dtype, T, cache):
    """More than 16 tiles of 64 keys a workgroup: looked up again, with a window that begins and blocks that are missing beyond that."""
    st = of_one([(60, 3001 - 13 * i) for i in range(10)] * 30, T=T, h=2, group=2, d=d, dtype=dtype, cache="e4m3" if cache == "e4m3" else None)
    assert units(st) >= SLOTS and tiles(min(s[2] for s in st.seqs)) > 2 * 16
    gone(st, 40, 1030 // T, 2100 // T, 2600 // T)
    check(st, window)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (80, "fp16"), (96, "bf16"), (112, "fp16"), (128, "bf16")])
@pytest.mark.parametrize("seqs,h", [([(40, 5000)], 1), ([(20, 2100), (300, 3000)], 4)])
def test_many_queries_split(seqs, h, d, dtype, T, cache):
    """Sequences split in tiles of 128 rows, joined a workgroup a row and (more than 4,096 rows) a wavefront a row."""
    st = of_one(seqs, T=T, h=h, group=4, d=d, dtype=dtype, cache="e4m3" if cache == "e4m3" else None)
    assert units(st) < 64 and (st.rows * st.hq > 4096) == (h == 4)
    check(st)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("n_new", [1, 9, 40])
def test_more_than_64_sequences(n_new, cache):
    """Beyond 64 sequences the plan is an even share: most stay whole, the long ones are split; the last are found behind the first 64."""
    seqs = [(n_new, n_new + 11 * i) for i in range(130)]
    seqs[3] = seqs[100] = seqs[129] = (n_new, 30000)
    st = of_one(seqs, h=2, group=2, d=128, cache="e4m3" if cache == "e4m3" else None)
    work = sum(-(-a * 2 // 16) * tiles(b) for a, b in seqs)
    assert tiles(30000) > 4 * work / SLOTS
    check(st)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_many_queries_in_a_graph(cache):
    """A step of a split chunk and whole ones, replayed with the work memory and the output used by others between, beside eager calls."""
    st = of_one([(70, 4000), (33, 33), (100, 100)], h=2, group=4, d=128, cache="e4m3" if cache == "e4m3" else None).to_gpu()
    out = torch.empty((st.rows, st.hq, st.d), dtype=ref.TYPES[st.dtype], device=DEV)
    lse = torch.empty((st.rows, st.hq), device=DEV)
    attn = B.make_attn(st.hq, B.BF16, 0.1)
    work = torch.empty(B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn), dtype=torch.uint8, device=DEV)

    def step():
        B.tutti_kv_attend(st.pool, st.scales, st.batch, attn, B.make_rows(st.d_q), B.make_rows(out), lse, work, work.numel())

    step()
    torch.cuda.synchronize()
    want, want_lse = out.clone(), lse.clone()
    assert bool(torch.isfinite(want.float()).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        out.fill_(i)
        lse.fill_(i)
        work.fill_(17 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        out.fill_(-1)
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
