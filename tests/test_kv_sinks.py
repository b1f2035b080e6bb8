"""Attention over a window and the first tokens, tutti_kv_attend_sinks: against 64-bit definitions on the GPU, and what it refuses
(CPU)."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
import sinks_reference
from paper_2605_03375_amd import binding as B
from test_kv_ops import BAD_POOLS, DEV, FAKE, SCALES, Step, _append_args, _code, run_attend, same

gpu = pytest.mark.gpu
DTYPE = {"bf16": B.BF16, "fp16": B.FP16}


def without_hidden(st, window, sinks):
    """Blocks of which no query sees a key leave the table: they have been given back."""
    for _, n_new, n_held, off in st.seqs:
        first = max(0, n_held - n_new + 1 - window) if window else 0
        for n in range(-(-n_held // st.T)):
            if n * st.T >= sinks and (n + 1) * st.T <= first:
                st.table[off + n] = B.NO_BLOCK


def run_sinks(st, window, sinks, sm_scale=None, work_fill=0xff):
    out = torch.full((max(1, st.rows), st.hq, st.d), math.nan, dtype=ref.TYPES[st.dtype], device=DEV)
    lse = torch.full((max(1, st.rows), st.hq), math.nan, device=DEV)
    attn = B.make_attn(st.hq, DTYPE[st.dtype], 1.0 / math.sqrt(st.d) if sm_scale is None else sm_scale, window=window)
    need = B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn)
    work = torch.full((need,), work_fill, dtype=torch.uint8, device=DEV)
    B.tutti_kv_attend_sinks(st.pool, st.scales, st.batch, attn, sinks, B.make_rows(st.d_q), B.make_rows(out), lse, work, need, st.status)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy(), int(st.status.item())


def check_sinks(st, window, sinks, sm_scale=None, table_len=None):
    """Every output within the error that the stated roundings allow."""
    out, lse, status = run_sinks(st.to_gpu() if table_len is None else st, window, sinks, sm_scale)
    want, want_lse, err, lse_err, want_status = sinks_reference.attend(
        st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 1.0 / math.sqrt(st.d) if sm_scale is None else sm_scale, window, sinks, table_len)
    assert status == want_status
    untouched = np.isnan(want_lse)
    assert np.array_equal(np.isnan(out), np.broadcast_to(untouched[:, :, None], out.shape) | np.isnan(want))
    fine = np.isfinite(want)
    assert np.array_equal(out[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    over = np.abs(out[fine] - want[fine]) - err[fine]
    assert over.size == 0 or over.max() <= 0, f"{over.max():.3g} beyond the bound"
    none = want_lse == -math.inf
    assert np.array_equal(lse == -math.inf, none) and np.array_equal(np.isnan(lse), untouched)
    fine = np.isfinite(want_lse)
    assert (np.abs(lse[fine] - want_lse[fine]) <= lse_err[fine]).all()
    return out, lse


SHAPES = [
    [(1, 1)], [(1, 2)], [(1, 33)], [(1, 300)], [(1, 1000)], [(3, 3)], [(5, 64)], [(8, 700)], [(20, 200)], [(33, 33)], [(70, 300)], [(130, 131)],
    [(300, 300)], [(64, 900)], [(0, 0), (1, 20), (0, 9)], [(1, 1 + 37 * i) for i in range(70)],
    [(1, 3000), (90, 200), (7, 7), (1, 1), (33, 1033)]]


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("seqs", SHAPES, ids=lambda s: "-".join(f"{a}of{b}" for a, b in s[:5]))
def test_lengths(seqs, group, cache):
    st = Step(seqs, group=group, cache="e4m3" if cache == "e4m3" else None, seed=len(seqs))
    without_hidden(st, 50, 5)
    check_sinks(st, 50, 5)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("window,sinks", [
    (1, 1), (1, 16), (2, 31), (31, 32), (32, 33), (33, 17), (64, 64), (64, 65), (100, 128), (17, 200), (200, 4), (4096, 4), (1, 1000), (40, 960),
    (50, 1 << 31), (3, 0xffffffff)])
def test_windows_and_first_tokens(window, sinks, cache):
    """Tiles with first tokens alone, with both, one that holds the end of the former and the begin of the window, and neither."""
    for seqs in ([(1, 1000), (1, 40)], [(6, 333), (16, 460)], [(150, 400), (1, 200), (40, 40)]):
        st = Step(seqs, cache="e4m3" if cache == "e4m3" else None, seed=window)
        without_hidden(st, window, sinks)
        check_sinks(st, window, sinks)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T,h,group,d,hnd,dtype,gap", [
    (16, 8, 4, 128, False, "bf16", 0), (16, 8, 4, 128, True, "fp16", 0), (32, 1, 8, 128, True, "bf16", 48), (64, 5, 1, 80, False, "bf16", 0),
    (64, 2, 1, 80, True, "fp16", 16), (16, 3, 2, 112, False, "bf16", 0), (1, 2, 3, 16, False, "fp16", 0), (5, 4, 1, 96, True, "bf16", 16),
    (48, 2, 2, 64, False, "bf16", 0), (24, 1, 8, 128, False, "fp16", 0), (128, 1, 2, 64, False, "bf16", 0), (12, 2, 8, 32, False, "bf16", 0)])
def test_layouts(cache, T, h, group, d, hnd, dtype, gap):
    kind = "e4m3" if cache == "e4m3" else None
    for seqs in ([(1, 300), (3, 130), (2, 2)], [(100, 300), (1, 130), (9, 9)]):
        st = Step(seqs, T=T, h=h, group=group, d=d, dtype=dtype, hnd=hnd, gap=gap, pad_rows=2, cache=kind, seed=T + d)
        without_hidden(st, 70, 21)
        check_sinks(st, 70, 21)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 10])
@pytest.mark.parametrize("seqs,window,sinks", [([(1, 9000)], 6000, 700), ([(1, 5000), (1, 4000)], 2500, 1), ([(4, 7000)], 5000, 64),
                                               ([(40, 6000)], 4000, 300)])
def test_keys_in_many_parts(seqs, window, sinks, T, cache):
    """Sequences that are split: parts with first tokens, with both, with the window's alone; few rows and many."""
    st = Step(seqs, T=T, h=1, group=4, d=128, cache="e4m3" if cache == "e4m3" else None)
    without_hidden(st, window, sinks)
    check_sinks(st, window, sinks)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("n,held,window,sinks,h", [(150, lambda i: 40 + 13 * i, 90, 7, 2), (65, lambda i: 1500, 1100, 40, 1),
                                                   (130, lambda i: 900, 700, 4, 4), (100, lambda i: 17 + 29 * i, 1300, 33, 3),
                                                   (300, lambda i: 1 + i * i % 700, 400, 100, 4), (700, lambda i: 1 + i % 500, 300, 5, 4)])
def test_more_sequences_than_lanes(n, held, window, sinks, h, cache):
    """Records beyond the first 64, of one length and of many: row tiles whole and in parts, as many as there is work memory for."""
    st = Step([(1 + i % 2 if n == 150 else 1, held(i) + 1) for i in range(n)], h=h, group=2, d=64, cache="e4m3" if cache == "e4m3" else None)
    without_hidden(st, window, sinks)
    check_sinks(st, window, sinks)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 12])
def test_blocks_that_are_not_there(T, cache):
    """Missing blocks among the first tokens and in the window are reported, and their keys not seen; a row may see none."""
    kind = "e4m3" if cache == "e4m3" else None
    for seqs in ([(1, 500), (1, 10)], [(3, 290), (40, 200)]):
        for at in (0, 1, -1, -2):
            st = Step(seqs, T=T, cache=kind)
            n = -(-seqs[0][1] // T)
            st.table[at % n] = (st.blocks, B.NO_BLOCK)[at % 2]
            check_sinks(st, 100, 20)
        st = Step(seqs, T=T, cache=kind)
        st.to_gpu()
        st.set_batch(table_len=len(st.table) - 2)
        check_sinks(st, 100, 20, table_len=len(st.table) - 2)
    st = Step([(1, 400), (9, 90)], T=T, cache=kind)
    st.table[:] = B.NO_BLOCK
    out, lse = check_sinks(st, 50, 4)
    assert (out == 0).all() and (lse == -math.inf).all()


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 10])
@pytest.mark.parametrize("n_new", [1, 5, 60])
def test_values_that_are_not_finite(T, n_new, cache):
    """An infinity or NaN among the values, in front of, among and behind the first tokens, in the same tile as they, or in the window:
    the queries that see it have it, no others do."""
    for at in (2, 6, 9, 17, 40, 190, 199, 199 + n_new // 2):
        st = Step([(n_new, 200 + n_new)], T=T, cache="e4m3" if cache == "e4m3" else None, d=128)
        st.cpu.planes[1][st.table[at // T], at % T, 1, 7] = 0x7f if cache == "e4m3" else math.inf
        out, lse = check_sinks(st, 12, 7)
        places = 200 + np.arange(n_new)
        sees = (at <= places) & ((at > places - 12) | (at < 7))
        hit = sees[:, None] & (np.arange(st.hq) // st.group == 1)
        assert np.array_equal(~np.isfinite(out[:, :, 7]), hit) and np.isfinite(np.delete(out, 7, 2)).all()
        # keys: a NaN makes whole rows NaN, where they see it
        st = Step([(n_new, 200 + n_new)], T=T, cache="e4m3" if cache == "e4m3" else None, d=128)
        st.cpu.planes[0][st.table[at // T], at % T, 0, 3] = 0x7f if cache == "e4m3" else math.nan
        out, _, _ = run_sinks(st.to_gpu(), 12, 7)
        hit = np.broadcast_to((sees[:, None] & (np.arange(st.hq) // st.group == 0))[:, :, None], out.shape)
        assert np.array_equal(np.isnan(out), hit), at


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_scores_that_are_large_or_negative_or_nothing(cache):
    kind = "e4m3" if cache == "e4m3" else None
    for sm_scale, spread in ((0.0, 1.0), (-1.5, 1.0), (0.3, 6.0)):
        for seqs in ([(1, 700), (6, 190)], [(70, 300)]):
            check_sinks(Step(seqs, cache=kind, spread=spread), 60, 40, sm_scale)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_nothing_to_add_is_the_plain_call(cache):
    """No first tokens, or no window: the bits of tutti_kv_attend."""
    for seqs in ([(1, 900), (2, 40)], [(130, 400)]):
        for window, sinks in ((0, 0), (0, 5), (100, 0)):
            st = Step(seqs, cache="e4m3" if cache == "e4m3" else None).to_gpu()
            a, b = run_attend(st, window=window), run_sinks(st, window, sinks)
            assert same(a[0], b[0]) and same(a[1], b[1]) and a[2] == b[2] == 0


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_records_that_cannot_be_honoured(cache):
    for bad in [(5, 4, 3, 0), (38, 5, 20, 0), (0, 31, 40, 0), (0, 1, 0x80000000, 0), (0xffffffff, 1, 1, 0)]:
        st = Step([(10, 120), (30, 130)], cache="e4m3" if cache == "e4m3" else None)
        st.seqs = [st.seqs[0], bad, st.seqs[1]]
        st.to_gpu()
        st.set_batch(max_new=30)
        out, lse, status = run_sinks(st, 20, 5)
        assert status == B.ST_BAD_EXTENT, bad
        st.seqs = [st.seqs[0], st.seqs[2]]
        want, _, err, _, _ = sinks_reference.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 1.0 / math.sqrt(st.d), 20, 5)
        assert (np.abs(out - want) <= err).all()


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("n_new", [1, 9, 70])
@pytest.mark.parametrize("window,sinks", [(300, 70), (40, 4), (2100, 700)])
def test_streams_of_two_thousand_million_tokens(window, sinks, n_new, cache):
    """Close to 2^31 tokens held, all but the seen ones given back: the bits of a short sequence with the same blocks.  (Places in tiles and
    blocks are the same, and windows say how the keys are split.)"""
    T, far = 256, (1 << 31) - (1 << 13)
    st = Step([(n_new, 4096 + 77)], T=T, h=2, group=2, d=64, cache="e4m3" if cache == "e4m3" else None).to_gpu()
    near = run_sinks(st, window, sinks)
    held = far + 77
    table = torch.full((-(-held // T),), -1, dtype=torch.int32, device=DEV)
    first = -(-sinks // T)
    table[:first] = st.d_table[:first]
    last = 4096 // T - first + 1
    table[-last:] = st.d_table[-last:]
    seqs = torch.tensor([[0, n_new, held, 0]], dtype=torch.int32, device=DEV)
    st.batch = B.make_batch(seqs, 1, n_new, table, table.numel(), st.rows)
    again = run_sinks(st, window, sinks)
    assert same(near[0], again[0]) and same(near[1], again[1]) and near[2] == again[2] == 0 and np.isfinite(near[0]).all()


@gpu
def test_rows_that_no_sequence_has():
    """So many that workgroups of one head would be too many for a launch, and those of four are not: the same results."""
    st = Step([(1, 700), (1, 90)], h=8, group=1, d=64).to_gpu()
    want = run_sinks(st, 100, 5)
    n = 1 << 26
    attn = B.make_attn(st.hq, B.BF16, 1.0 / math.sqrt(st.d), window=100)
    batch = B.make_batch(st.d_seqs, 2, 1, st.d_table, st.d_table.numel(), n)
    out, lse = torch.empty((st.rows, st.hq, st.d), dtype=torch.bfloat16, device=DEV), torch.empty((st.rows, st.hq), device=DEV)
    work = torch.empty(B.tutti_kv_attend_work_bytes(st.pool, batch, attn), dtype=torch.uint8, device=DEV)
    B.tutti_kv_attend_sinks(st.pool, None, batch, attn, 5, B.make_rows(st.d_q), B.make_rows(out), lse, work, work.numel(), st.status)
    torch.cuda.synchronize()
    ref_out, ref_lse, err, lse_err, _ = sinks_reference.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, 1, 1.0 / math.sqrt(st.d), 100, 5)
    for got_out, got_lse in ((out.float().cpu().numpy(), lse.cpu().numpy()), want[:2]):
        assert (np.abs(got_out - ref_out) <= err).all() and (np.abs(got_lse - ref_lse) <= lse_err).all()
    assert int(st.status.item()) == 0


@gpu
def test_twice_the_same_on_another_stream_and_in_a_graph():
    st = Step([(1, 3000), (1, 500), (2, 400)], h=8, d=128, cache="e4m3").to_gpu()
    want = run_sinks(st, 1500, 100)
    for fill in (0x00, 0x7f, 0x3c):
        again = run_sinks(st, 1500, 100, work_fill=fill)
        assert same(want[0], again[0]) and same(want[1], again[1])
    out = torch.empty((st.rows, st.hq, st.d), dtype=torch.bfloat16, device=DEV)
    lse = torch.empty((st.rows, st.hq), device=DEV)
    attn = B.make_attn(st.hq, B.BF16, 1.0 / math.sqrt(st.d), window=1500)
    work = torch.empty(B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn), dtype=torch.uint8, device=DEV)

    def step():
        B.tutti_kv_attend_sinks(st.pool, st.scales, st.batch, attn, 100, B.make_rows(st.d_q), B.make_rows(out), lse, work, work.numel())

    def check():
        torch.cuda.synchronize()
        assert same(out.float().cpu().numpy(), want[0]) and same(lse.cpu().numpy(), want[1])

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        out.fill_(i)
        work.fill_(17 * i)
        graph.replay()
        check()
        step()
        check()


# ---------------------------------------------------------------- refusals (CPU)

def test_refuses():
    def args(**kw):
        pool, scales, batch, _, q, out, *_ = _append_args(**{k: v for k, v in kw.items() if k != "attn"})
        attn = B.make_attn(4, kw.get("dtype", B.BF16), 0.1, window=8)
        for name, x in kw.get("attn", {}).items():
            setattr(attn, name, x)
        return pool, scales, batch, attn, 4, q, out, kw.get("lse", 0), kw.get("work", FAKE), kw.get("bytes", 1 << 40), kw.get("status", 0)

    assert _code(B.tutti_kv_attend_sinks, *args()) == B.OK
    bad = [dict(pool=p) for p in BAD_POOLS] + [
        dict(scales=SCALES), dict(dtype=0), dict(attn=dict(n_q_heads=0)), dict(attn=dict(n_q_heads=5)), dict(attn=dict(sm_scale=math.inf)),
        dict(attn=dict(causal=2)), dict(attn=dict(causal=0)), dict(lse=FAKE + 2), dict(status=FAKE + 1),
        dict(batch=dict(n_seq=1, d_seqs=FAKE + 4)), dict(batch=dict(n_seq=1), work=0), dict(batch=dict(n_seq=1), work=FAKE + 8),
        dict(rows=dict(q=B.make_rows(FAKE, 1000, 128))), dict(rows=dict(q_out=None))]
    for kw in bad:
        assert _code(B.tutti_kv_attend_sinks, *args(**kw)) == B.EINVAL, kw
    pool, _, batch, attn, *_ = args(batch=dict(n_seq=1))
    need = B.tutti_kv_attend_work_bytes(pool, batch, attn)
    assert need > 0 and _code(B.tutti_kv_attend_sinks, *args(batch=dict(n_seq=1), bytes=need - 1)) == B.ERANGE
    assert _code(B.tutti_kv_attend_sinks, *args(batch=dict(n_seq=B.MAX_REQ + 1))) == B.ERANGE
    for none in (0, 2, 3, 5, 6):
        call = list(args())
        call[none] = None
        assert _code(B.tutti_kv_attend_sinks, *call) == B.EINVAL


def test_the_reference_is_attention_with_a_window_where_there_are_no_first_tokens():
    st = Step([(3, 90), (1, 40)])
    a = ref.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 0.2, window=30)
    b = sinks_reference.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 0.2, 30, 0)
    assert all(np.array_equal(x, y) for x, y in zip(a[:4], b[:4]))
    a = ref.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 0.2)
    b = sinks_reference.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 0.2, 30, 90)
    assert all(np.array_equal(x, y) for x, y in zip(a[:4], b[:4]))
