"""Tables, counts and pools that tutti_blocks_* can meet beside those of test_blocks: entries that name free blocks, and sizes at which every
loop of a kernel goes round again.  On the GPU, against the definitions, to the last bit."""
import math
import random

import numpy as np
import pytest
import torch

import blocks_reference as ref
import kv_reference
import sinks_reference
from paper_2605_03375_amd import binding as B
from test_blocks import DEV, NONE, Pool, back, both, gpu, random_pool, words
from test_kv_ops import make_angles


# ---------------------------------------------------------------- entries that name free blocks

def fork_from_used(uses, table, records, max_entries, max_pairs):
    """ref.fork, where sources' entries that name a block without uses are taken as entries that name none."""
    stale = [b < len(uses) and uses[b] == 0 for b in table]
    named = [NONE if s else b for s, b in zip(stale, table)]
    mine, hit = list(named), False
    pairs, status = ref.fork(uses, mine, records, max_entries, max_pairs)
    written = set()
    for src, dst, shared, copied, new in records:
        hit |= any(stale[src:src + shared + copied])
        written.update(range(dst, dst + shared + copied + new))
    for e in range(len(table)):
        if e in written:
            table[e] = mine[e]
    return pairs, status | (B.ST_BAD_USES if hit else 0)


def check_fork(uses, table, records, pad=0):
    """The call against fork_from_used; returns the pairs."""
    records = records + [(0, 0, 0, 0, 0)] * pad
    p = Pool(uses, table)
    max_pairs, most = sum(r[3] for r in records), max([sum(r[2:]) for r in records] + [1])
    rec = np.zeros(len(records), B.FORK_DTYPE)
    for i, r in enumerate(records):
        rec[i] = (*r, (9, 9, 9))
    pairs, n_pairs = words([3] * (2 * max_pairs + 2)), words([3])
    need = B.tutti_blocks_fork_work_bytes(len(uses), len(records))
    work = torch.full((need + 16,), 0xff, dtype=torch.uint8, device=DEV)
    B.tutti_blocks_fork(p.d_uses, len(uses), p.d_table, len(table), words(rec.view(np.uint32)), len(records), most, pairs, n_pairs, max_pairs,
                        work, need, p.d_status)
    want, status = fork_from_used(p.uses, p.table, records, most, max_pairs)
    p.check(status)
    assert back(n_pairs) == [len(want)] and back(pairs) == [x for q in want for x in q] + [3, 3]
    assert bool((work[need:] == 0xff).all())
    return want, status


def test_the_reference_leaves_free_blocks_alone():
    """What goes wrong without: the free block that an entry names is handed out in the same call, and has two owners."""
    uses, table = [1, 0, 0, 1], [0, 1, 3] + [NONE] * 6
    a, b = list(uses), list(table)
    ref.fork(a, b, [(0, 3, 3, 0, 0), (0, 6, 0, 0, 2)], 3, 0)
    assert b[4] == b[6] == 1 and a[1] == 2
    a, b = list(uses), list(table)
    assert fork_from_used(a, b, [(0, 3, 3, 0, 0), (0, 6, 0, 0, 2)], 3, 0) == ([], B.ST_BAD_USES)
    assert b[:8] == [0, 1, 3, 0, NONE, 3, 1, 2] and a == [2, 1, 1, 2]


@gpu
@both
def test_fork_from_free_blocks(pad):
    uses, table = [1, 0, 0, 1, 0, 0], [0, 1, 3] + [NONE] * 20
    check_fork(uses, table, [(0, 3, 3, 0, 0), (0, 6, 0, 0, 2)], pad)                 # shared; handed out by the second record
    pairs, status = check_fork(uses, table, [(0, 3, 1, 2, 0), (0, 8, 0, 3, 1)], pad)   # copied: no pair has it as its source
    assert pairs == [(NONE, NONE), (3, 2), (0, 4), (NONE, NONE)] + [(NONE, NONE)] and status == B.ST_BAD_USES | B.ST_NO_FREE
    check_fork([0] * 6, [0, 1, 2, 3, 4, 5] + [NONE] * 20, [(0, 6, 3, 3, 0), (0, 12, 0, 6, 2)], pad)
    check_fork([2], [0, 0, 0] + [NONE] * 6, [(0, 3, 2, 1, 0)], pad)


@gpu
@pytest.mark.parametrize("blocks", [3, 64, 65, 1000, 65536, 65537, 70001, (1 << 20) + 1500])
@pytest.mark.parametrize("n_seq,width,pad", [(4, 64, 0), (4, 64, 1100), (70, 90, 0), (3, 1500, 0)])
def test_some_of_the_entries_name_free_blocks(blocks, n_seq, width, pad):
    """Both kernels; the pool's last blocks; neighbours that share; every word of the bits."""
    rng = np.random.default_rng(blocks)
    uses = (rng.random(blocks) < 0.8).astype(int) * rng.integers(1, 3, blocks)
    uses[-3:] = [0, 1, 0]
    table = rng.integers(0, blocks, n_seq * width)
    table[rng.random(table.size) < 0.1] = NONE
    table[::7] = blocks - 1 - np.arange(table[::7].size) % 3
    for i in range(1, n_seq, 3):
        table[i * width:i * width + width // 2] = table[(i - 1) * width:(i - 1) * width + width // 2]
    records = []
    for i in range(n_seq):
        n = int(rng.integers(0, width + 1))
        copied = int(min(n, rng.integers(0, 5)))
        records.append((i * width, (n_seq + i) * width, n - copied, copied, int(min(width - n, rng.integers(0, 3)))))
    check_fork(uses.tolist(), table.tolist() + [NONE] * (n_seq * width), records, pad)


def compact_used(uses, table, max_pairs):
    """ref.compact, after which entries that named a hole name no block."""
    n = sum(u != 0 for u in uses)
    holes = [e for e, b in enumerate(table) if b < n and uses[b] == 0]
    pairs, n, status = ref.compact(uses, table, max_pairs)
    for e in holes:
        table[e] = NONE
    return pairs, n, status | (B.ST_BAD_USES if holes else 0)


def check_compact(uses, table, max_pairs):
    p = Pool(uses, table)
    pairs, totals = words([3] * (2 * max_pairs + 2)), words([3, 3, 3])
    need = B.tutti_blocks_compact_work_bytes(len(uses))
    work = torch.full((need + 16,), 0xff, dtype=torch.uint8, device=DEV)
    B.tutti_blocks_compact(p.d_uses, len(uses), p.d_table, len(table), pairs, totals, max_pairs, work, need, p.d_status)
    want, n, status = compact_used(p.uses, p.table, max_pairs)
    p.check(status)
    assert back(totals) == [len(want), n, 3] and bool((work[need:] == 0xff).all())
    assert back(pairs) == [x for q in want for x in q] + [3] * (2 * (max_pairs - len(want)) + 2)
    return want, status


def test_the_reference_does_not_give_a_hole_s_entry_what_moves_there():
    uses, table = [1, 0, 0, 1], [0, 1, 2, 3]
    a, b = list(uses), list(table)
    ref.compact(a, b, 2)
    assert b[1] == b[3] == 1 and a[1] == 1                 # two entries, one use
    a, b = list(uses), list(table)
    assert compact_used(a, b, 2) == ([(3, 1)], 2, B.ST_BAD_USES) and b == [0, NONE, 2, 1]


@gpu
@pytest.mark.parametrize("blocks", [1, 2, 5, 64, 65, 1000, 1025, 40003, (1 << 20) + 1500])
def test_compact_with_entries_that_name_free_blocks(blocks):
    """Holes, whether something moves into them or not; free blocks behind the used ones; the pool's last blocks."""
    rng = np.random.default_rng(blocks)
    for share in (0.0, 0.03, 0.5, 0.97, 1.0):
        uses = ((rng.random(blocks) < share) * rng.integers(1, 4, blocks)).tolist()
        table = rng.integers(0, blocks, 3000)
        table[::9] = blocks - 1 - np.arange(table[::9].size) % min(blocks, 70)
        table[rng.random(table.size) < 0.1] = NONE
        for most in {0, 1, blocks // 5, blocks // 2}:
            check_compact(uses, table.tolist(), most)


# ---------------------------------------------------------------- sizes at which loops go round again

def follow(uses, table, max_pairs):
    """ref.compact for large pools: pairs, and uses and table as they are afterwards."""
    blocks = uses.size
    n = int((uses != 0).sum())
    holes, movers = np.flatnonzero(uses[:n] == 0), n + np.flatnonzero(uses[n:])[::-1]
    k = min(max_pairs, holes.size)
    holes, movers = holes[:k], movers[:k]
    to = np.arange(blocks)
    to[movers] = holes
    uses = uses.copy()
    uses[holes] = uses[movers]
    uses[movers] = 0
    named = table != NONE
    return np.stack([movers, holes], 1), n, uses, np.where(named, to[np.where(named, table, 0)], NONE)


def test_large_pools_follow_the_reference():
    rng = random.Random(3)
    uses, table, _ = random_pool(500, 12, 20, rng)
    for most in (0, 3, 250):
        pairs, n, u, t = follow(np.array(uses), np.array(table), most)
        a, b = list(uses), list(table)
        want, m, status = ref.compact(a, b, most)
        assert (pairs.tolist(), n, u.tolist(), t.tolist(), status) == ([list(p) for p in want], m, a, b, 0)


@gpu
@pytest.mark.parametrize("blocks,share,entries", [(2_000_003, 0.3, 5_000_001), (1_300_000, 0.55, 1_572_865), (600_001, 0.01, 3_200_000)])
def test_compaction_of_more_than_a_grid_takes_at_once(blocks, share, entries):
    """Tables of more than 1,572,864 entries, more than 524,288 blocks behind the used ones' end; thousands of chunks."""
    rng = np.random.default_rng(blocks)
    uses = (rng.random(blocks) < share) * rng.integers(1, 5, blocks)
    uses[-1] = 1
    used = np.flatnonzero(uses)
    table = used[rng.integers(0, used.size, entries)]
    table[rng.random(entries) < 0.05] = NONE
    table[-1] = table[0] = blocks - 1
    for most in (blocks // 2, 1000):
        d_uses, d_table, status = words(uses), words(table), torch.zeros(1, dtype=torch.int32, device=DEV)
        pairs, totals = words([3] * (2 * most)), words([3, 3])
        work = torch.full((B.tutti_blocks_compact_work_bytes(blocks),), 0xff, dtype=torch.uint8, device=DEV)
        B.tutti_blocks_compact(d_uses, blocks, d_table, entries, pairs, totals, most, work, work.numel(), status)
        torch.cuda.synchronize()
        want, n, u, t = follow(uses, table, most)
        assert totals.tolist() == [len(want), n] and int(status.item()) == 0
        assert torch.equal(pairs[:want.size].cpu(), words(want.ravel()).cpu()) and bool((pairs[want.size:] == 3).all())
        assert torch.equal(d_uses, words(u)) and torch.equal(d_table, words(t))


@gpu
@pytest.mark.parametrize("T,h,d,gap,blocks,n", [(16, 2, 64, 0, 12000, 5000),      # one piece of 4 KiB a block
                                                (10, 4, 128, 48, 8000, 3001),     # three pieces, the last one half
                                                (4096, 40, 128, 16, 5, 2),        # 10,240 pieces
                                                (1, 1, 16, 0, 30000, 14999)])     # two lanes' loads
def test_copies_of_more_than_a_grid_takes_at_once(T, h, d, gap, blocks, n):
    """Where the number of pairs lies on the device 8,192 pieces are copied at a time: each once, with its scales, and nothing else."""
    stride = T * h * d * 2 + gap
    assert 2 * n * -(-T * h * d * 2 // 4096) > 8192
    gen = torch.Generator(device=DEV)
    gen.manual_seed(n)
    planes = [torch.randint(-2 ** 62, 2 ** 62, (blocks * stride // 8,), generator=gen, device=DEV) for _ in range(2)]
    scales = [torch.randn(blocks, h + 2, device=DEV) for _ in range(2)]
    pool = B.make_pool(*planes, num_blocks=blocks, block_tokens=T, num_kv_heads=h, head_dim=d, elt_bytes=2, block_stride=stride)
    order = np.random.default_rng(n).permutation(blocks)
    pairs = np.stack([order[:n], order[n:2 * n]], 1)
    pairs[n // 2] = NONE
    real = np.delete(pairs, n // 2, 0)
    src, dst = (torch.from_numpy(real[:, i].astype(np.int64)).to(DEV) for i in range(2))
    size = (stride - gap) // 8
    want = [p.clone() for p in planes]
    for x in want:
        x = x.view(blocks, stride // 8)
        x[dst, :size] = x[src, :size]
    want_s = [s.clone() for s in scales]
    for x in want_s:
        x[dst, :h] = x[src, :h]
    spare = np.stack([order[2 * n:2 * n + 1], order[2 * n:2 * n + 1]], 1)      # behind what the device says there is
    d_pairs, status = words(np.concatenate([pairs, spare])), torch.zeros(1, dtype=torch.int32, device=DEV)
    B.tutti_blocks_copy(pool, B.make_scales(*scales), d_pairs, words([n]), len(pairs) + len(spare), status)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(planes + scales, want + want_s)) and int(status.item()) == 0


# ---------------------------------------------------------------- rotated streams

@gpu
def test_a_rotated_stream_outlives_its_pool():
    """200 tokens in a pool of 8 blocks, rotated by their places in the whole stream and not again: results are the definition's over all
    keys that were ever appended, rotated so; a token beyond the table of angles is refused."""
    T, h, hq, d, blocks, window, sinks, n = 16, 2, 4, 64, 8, 50, 5, 200
    rng = np.random.default_rng(4)
    angles = make_angles(n, d)
    rope = B.make_rope(torch.from_numpy(angles).to(DEV), d)
    planes = [torch.zeros(blocks * T * h * d, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    pool = B.make_pool(*planes, num_blocks=blocks, block_tokens=T, num_kv_heads=h, head_dim=d, elt_bytes=2)
    uses, table = torch.zeros(blocks, dtype=torch.int32, device=DEV), torch.full((16,), -1, dtype=torch.int32, device=DEV)
    work = torch.empty(B.tutti_blocks_fork_work_bytes(blocks, 1), dtype=torch.uint8, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    x = kv_reference.round16(rng.standard_normal((n + 1, hq + 2 * h, d)), "bf16")
    # all of it on the CPU: rotated keys and queries, and a cache that holds every block
    whole = kv_reference.Cache(13, T, h, d, "bf16")
    want_q, _ = kv_reference.append(whole, "bf16", [(0, n, n, 0)], np.arange(13, dtype=np.uint32), x[:n, :hq], x[:n, hq:hq + h], x[:n, hq + h:],
                                    dict(cos_sin=angles, rot=d, interleaved=False, pos=None, pairs=None), None)
    want, _, err, _, _ = sinks_reference.attend(whole, "bf16", [(0, n, n, 0)], np.arange(13, dtype=np.uint32), want_q, hq // h,
                                                1.0 / math.sqrt(d), window, sinks)
    for held in range(1, n + 2):
        if held % T == 1:
            gone = max(0, held - window) // T
            B.tutti_blocks_free(uses, blocks, table, 16, words([(1, max(0, gone - 1))]), 1, 16, status)
            rec = np.zeros(1, B.FORK_DTYPE)
            rec[0] = (0, held // T, 0, 0, 1, (0, 0, 0))
            B.tutti_blocks_fork(uses, blocks, table, 16, words(rec.view(np.uint32)), 1, 1, None, None, 0, work, work.numel(), status)
        row = torch.from_numpy(x[held - 1:held]).to(torch.bfloat16).to(DEV)
        q, out = torch.full((1, hq, d), math.nan, dtype=torch.bfloat16, device=DEV), torch.empty((1, hq, d), dtype=torch.bfloat16, device=DEV)
        batch = B.make_batch(words([(0, 1, held, 0)]), 1, 1, table, 16, 1)
        B.tutti_kv_append(pool, None, batch, rope, B.make_rows(row[:, :hq]), B.make_rows(q), B.make_rows(row[:, hq:hq + h]),
                          B.make_rows(row[:, hq + h:]), hq, B.BF16, status)
        if held > n:
            break
        attn = B.make_attn(hq, B.BF16, 1.0 / math.sqrt(d), window=window)
        more = torch.empty(B.tutti_kv_attend_work_bytes(pool, batch, attn), dtype=torch.uint8, device=DEV)
        B.tutti_kv_attend_sinks(pool, None, batch, attn, sinks, B.make_rows(q), B.make_rows(out), None, more, more.numel(), status)
        assert np.array_equal(q.float().cpu().numpy()[0], want_q[held - 1])
        assert (np.abs(out.float().cpu().numpy()[0] - want[held - 1]) <= err[held - 1]).all(), held
    assert int(status.item()) == B.ST_BAD_POS and bool(torch.isnan(q).all())
