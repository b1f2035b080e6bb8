"""Blocks that are shared, copied, given back and moved (tutti_blocks_*): against their definitions on the GPU, all of it to the last bit;
together with appending and attention; and what the calls refuse (CPU)."""
import math
import random

import numpy as np
import pytest
import torch

import blocks_reference as ref
import kv_reference
from paper_2605_03375_amd import binding as B

DEV = "cuda:0"
FAKE = 0x10000
NONE = B.NO_BLOCK
gpu = pytest.mark.gpu


def words(x):
    return torch.from_numpy(np.asarray(x, np.uint32).view(np.int32).copy()).to(DEV)


def back(t):
    return [int(x) for x in t.cpu().numpy().view(np.uint32).ravel()]


class Pool:
    """Counts and a table on both sides; 16 entries behind either end of the table's memory that nobody may touch."""

    def __init__(self, uses, table):
        self.uses, self.table = [int(u) for u in uses], [int(t) for t in table]
        self.d_uses = words(self.uses + [7] * 5)
        self.d_all = words([5] * 16 + self.table + [5] * 16)
        self.d_table = self.d_all[16:16 + len(self.table)]
        self.d_status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def check(self, status):
        torch.cuda.synchronize()
        uses = back(self.d_uses)
        assert uses[len(self.uses):] == [7] * 5 and uses[:len(self.uses)] == self.uses
        got = back(self.d_all)
        assert got[:16] == got[-16:] == [5] * 16 and got[16:-16] == self.table
        assert int(self.d_status.item()) == status

    def fork(self, records, max_entries=None, max_pairs=None, work_fill=0xff, pad=0):
        """pad: so many records without entries behind these (over 1,024 records in all, two launches do what one does else)."""
        records = records + [(0, 0, 0, 0, 0)] * pad
        if max_entries is None:
            max_entries = max([s + c + n for _, _, s, c, n in records] + [1])
        if max_pairs is None:
            max_pairs = sum(r[3] for r in records)
        rec = np.zeros(len(records), B.FORK_DTYPE)
        for i, r in enumerate(records):
            rec[i] = (*r, (9, 9, 9))
        d_rec = words(rec.view(np.uint32)) if records else None
        pairs, n_pairs = words([3] * (2 * max_pairs + 2)), words([3])
        need = B.tutti_blocks_fork_work_bytes(len(self.uses), len(records))
        work = torch.full((need + 16,), work_fill, dtype=torch.uint8, device=DEV)
        B.tutti_blocks_fork(self.d_uses, len(self.uses), self.d_table, len(self.table), d_rec, len(records), max_entries, pairs, n_pairs,
                            max_pairs, work, need, self.d_status)
        want, status = ref.fork(self.uses, self.table, records, max_entries, max_pairs)
        self.check(status)
        assert back(n_pairs) == [len(want)]
        assert back(pairs) == [x for p in want for x in p] + [3] * (2 * (max_pairs - len(want)) + 2)
        assert bool((work[need:] == work_fill).all())
        return want, status

    def free(self, ranges, max_entries=None):
        max_entries = max([n for _, n in ranges] + [0]) if max_entries is None else max_entries
        B.tutti_blocks_free(self.d_uses, len(self.uses), self.d_table, len(self.table), words(ranges), len(ranges), max_entries,
                            self.d_status)
        status = ref.free(self.uses, self.table, ranges, max_entries)
        self.check(status)
        return status

    def compact(self, max_pairs=None, work_fill=0xff):
        max_pairs = len(self.uses) // 2 if max_pairs is None else max_pairs
        pairs, totals = words([3] * (2 * max_pairs + 2)), words([3, 3, 3])
        need = B.tutti_blocks_compact_work_bytes(len(self.uses))
        work = torch.full((need + 16,), work_fill, dtype=torch.uint8, device=DEV)
        B.tutti_blocks_compact(self.d_uses, len(self.uses), self.d_table, len(self.table), pairs, totals, max_pairs, work, need,
                               self.d_status)
        want, n, status = ref.compact(self.uses, self.table, max_pairs)
        self.check(status)
        assert back(totals) == [len(want), n, 3]
        assert back(pairs) == [x for p in want for x in p] + [3] * (2 * (max_pairs - len(want)) + 2)
        assert bool((work[need:] == work_fill).all())
        return want, status


def random_pool(blocks, n_seq, width, rng, share=0.5, halves=2):
    """Sequences of up to `width` blocks, some of whose first ones are shared; a second table behind the first; some blocks held by
    others."""
    order = rng.sample(range(blocks), blocks)
    uses, table, lengths, at = [0] * blocks, [NONE] * (halves * n_seq * width), [], 0
    for i in range(n_seq):
        n = rng.randint(1, width)
        shared = min(n, lengths[-1]) // 2 if lengths and rng.random() < share else 0
        for e in range(n):
            b = table[(i - 1) * width + e] if e < shared else order[at % (blocks // 2)]
            at += e >= shared
            table[i * width + e] = b
            if b != NONE:
                uses[b] += 1
        lengths.append(n)
    for b in order[-(blocks // 8):]:
        uses[b] = max(uses[b], 1)
    return uses, table, lengths


# ---------------------------------------------------------------- fork

both = pytest.mark.parametrize("pad", [0, 1100])


@gpu
@pytest.mark.parametrize("blocks", [1, 2, 3, 4, 5, 1023, 1024, 1025, 4099, 16384, 16390, 65533, 65536, 65537, 70001])
@pytest.mark.parametrize("most", [800, 1300])
def test_new_blocks_are_the_lowest_free_ones(blocks, most):
    """One launch (up to 65,536 blocks and 4,096 entries) and two."""
    rng = random.Random(blocks)
    for free_share in (0.0, 0.003, 0.02, 0.5, 1.0):
        p = Pool([0 if rng.random() < free_share else rng.randint(1, 3) for _ in range(blocks)], [NONE] * 3000)
        p.fork([(0, 0, 0, 0, 1), (0, 1, 0, 0, 0), (0, 1, 0, 0, 7), (0, 100, 0, 0, most), (0, 2000, 0, 0, 700)])


@gpu
@pytest.mark.parametrize("n,entries", [(4096 // 8, 8), (1, 4096), (1, 4097), (1024, 4), (1025, 3), (1000, 1)])
def test_records_at_the_ends_of_what_one_launch_does(n, entries):
    rng = random.Random(n)
    uses, table, lengths = random_pool(20000, 30, 20, rng, halves=1)
    off = len(table)
    records = [(rng.randrange(29) * 20, off + i * entries, c, min(entries - c, rng.randint(0, 2)), 0) for i in range(n)
               for c in [rng.randint(0, min(entries, 20))]]
    records = [(a, b, c, d, entries - c - d) if i % 3 else (a, b, c, d, 0) for i, (a, b, c, d, _) in enumerate(records)]
    Pool(uses, table + [NONE] * (n * entries)).fork(records)


@gpu
@pytest.mark.parametrize("n_seq,width", [(1, 1), (1, 3), (4, 64), (70, 33), (3, 1500), (300, 9), (2048, 2)])
def test_sequences_go_on_from_others(n_seq, width):
    rng = random.Random(n_seq)
    uses, table, lengths = random_pool(max(64, 4 * n_seq * width), n_seq, width, rng)
    records = []
    for i in range(n_seq):
        source = rng.randrange(n_seq)
        n = rng.randint(0, lengths[source])
        copied = min(n, rng.choice((0, 1, 1, 2, n)))
        records.append((source * width, (n_seq + i) * width, n - copied, copied, rng.randint(0, width - n)))
    for fill, pad in ((0xff, 0), (0, 0), (0, min(1100, 2048 - n_seq))):
        Pool(uses, table).fork(records, work_fill=fill, pad=pad)


@gpu
@both
def test_groups_that_share_their_blocks(pad):
    """Neighbours that name the same block at the same place, and some that do not; a source that names one block everywhere."""
    rng = random.Random(8)
    width = 40
    prefix = rng.sample(range(500), 60)
    table = [prefix[e] if e < 30 else 500 + i * width + e for i in range(20) for e in range(width)] + [NONE] * (40 * width)
    table[7 * width:8 * width] = [3] * width
    table[3 * width + 5], table[12 * width + 5] = NONE, 77
    uses = [0] * 3000
    for b in table:
        if b != NONE:
            uses[b] += 1
    p = Pool(uses, table)
    p.fork([((i if i % 5 else 7) * width, (20 + i) * width, width - 2 - i % 3, i % 3, i % 2) for i in range(20)], pad=pad)
    p.free([(i * width, width - i % 4) for i in range(40)])
    p.free([(i * width, width) for i in range(60)])


@gpu
def test_pools_of_more_spans_than_one_chunk_each():
    """Over 1,024 chunks of 1,024 blocks: spans of two chunks."""
    blocks = (1 << 20) + 1500
    rng = np.random.default_rng(0)
    uses = (rng.random(blocks) < 0.7).astype(np.uint32)
    uses[-3000:] = 0
    free = int((uses == 0).sum())
    p = Pool(uses, [NONE] * (free + 10))
    _, status = p.fork([(0, 0, 0, 0, free // 2), (0, free // 2, 0, 0, free - free // 2 + 10)])
    assert status == B.ST_NO_FREE
    q = Pool(uses, np.flatnonzero(uses)[::-1])
    q.compact()
    q.compact()


@gpu
@both
def test_entries_without_a_block(pad):
    """None, and ids beyond the pool: shared and copied as none; what is numbered for them stays free."""
    uses = [1, 1, 0, 0, 2, 0, 0, 1]
    table = [0, NONE, 1, 8, 4, NONE, 7, 0x80000000] + [NONE] * 24
    p = Pool(uses, table)
    assert p.fork([(0, 8, 4, 4, 2)], pad=pad)[1] == B.ST_BAD_BLOCK | B.ST_NO_FREE
    p = Pool(uses, table)
    pairs, _ = p.fork([(0, 8, 1, 2, 0), (4, 16, 0, 2, 1)], pad=pad)
    assert pairs == [(NONE, NONE), (1, 3), (4, 5), (NONE, NONE)]
    p = Pool([3, 2], [0, 1, 0, NONE] + [NONE] * 8)       # nothing is free
    assert p.fork([(0, 4, 1, 2, 1)], pad=pad)[0] == [(NONE, NONE)] * 2


@gpu
@both
def test_records_that_do_not_fit(pad):
    uses, table = [1] * 10 + [0] * 50, list(range(10)) + [NONE] * 30
    for bad in [(35, 10, 4, 2, 0), (0, 36, 4, 0, 1), (0xffffffff, 10, 1, 0, 0), (0, 0xffffffff, 0, 0, 1), (0, 10, 0xffffffff, 1, 0),
                (0, 10, 0x80000000, 0x80000000, 1), (0, 10, 0, 0, 0xffffffff), (0, 10, 3, 2, 2)]:
        p = Pool(uses, table)
        assert p.fork([(0, 20, 2, 1, 0), bad, (4, 25, 1, 1, 3)], max_entries=6, max_pairs=9, pad=pad)[1] == B.ST_BAD_EXTENT, bad
    p = Pool(uses, table)
    assert p.fork([(0xffffffff, 12, 0, 0, 2)], pad=pad)[1] == 0       # (a source that is not used)
    for max_pairs, kept in ((0, 0), (1, 1), (2, 1), (3, 3), (4, 4)):
        p = Pool(uses, table)
        pairs, status = p.fork([(0, 10, 2, 1, 0), (3, 15, 0, 2, 1), (5, 20, 1, 1, 0), (8, 25, 2, 0, 2)], max_pairs=max_pairs, pad=pad)
        assert (len(pairs), status) == (kept, 0 if max_pairs == 4 else B.ST_BAD_EXTENT)
    p = Pool(uses, table)
    p.fork([], pad=pad)
    p.fork([(0, 10, 0, 0, 0)], max_entries=0, pad=pad)
    assert p.fork([(0, 10, 1, 0, 0)], max_entries=0, pad=pad)[1] == B.ST_BAD_EXTENT


# ---------------------------------------------------------------- free

@gpu
@pytest.mark.parametrize("n_seq,width", [(1, 1), (5, 3), (70, 33), (4, 2500), (2048, 3)])
def test_free(n_seq, width):
    rng = random.Random(width)
    uses, table, lengths = random_pool(max(64, 4 * n_seq * width), n_seq, width, rng, halves=1)
    p = Pool(uses, table)
    ranges = []
    for i in range(n_seq):
        a = rng.randint(0, lengths[i])
        ranges.append((i * width + a, rng.randint(0, lengths[i] - a)))
    assert p.free(ranges) == 0
    assert p.free(ranges) == 0              # (there is nothing any more)
    p.free([(i * width, n) for i, n in enumerate(lengths)])


@gpu
def test_free_what_is_not_there_or_not_used_or_named_twice():
    uses = [2, 0, 1, 5]
    p = Pool(uses, [0, 1, 2, 3, 4, NONE, 0x7fffffff, 0, 0, 2])
    assert p.free([(0, 10)]) == B.ST_BAD_BLOCK | B.ST_BAD_USES
    p = Pool([64] * 8, [e % 8 for e in range(4096)])         # 512 releases of blocks with 64 uses
    assert p.free([(0, 4096)]) == B.ST_BAD_USES
    assert p.uses == [0] * 8
    p = Pool([9] * 8, [e % 8 for e in range(40)])            # entries in several ranges go once
    assert p.free([(0, 30), (10, 20), (10, 30), (0, 1)]) == 0
    assert p.uses == [4] * 8
    for bad in [(39, 2), (41, 0), (0xffffffff, 1), (0, 0xffffffff), (0, 31)]:
        p = Pool([9] * 8, [e % 8 for e in range(40)])
        assert p.free([(0, 3), bad, (10, 20)], max_entries=30) == B.ST_BAD_EXTENT, bad
    p = Pool([9] * 8, [e % 8 for e in range(40)])
    assert p.free([(3, 0), (40, 0)]) == 0 and p.free([(3, 1)], max_entries=0) == B.ST_BAD_EXTENT


# ---------------------------------------------------------------- compact

@gpu
@pytest.mark.parametrize("blocks", [1, 2, 3, 4, 7, 1023, 1024, 1025, 5000, 40003])
def test_compact(blocks):
    rng = random.Random(blocks)
    for share in (0.0, 0.03, 0.5, 0.97, 1.0):
        uses = [rng.randint(1, 4) if rng.random() < share else 0 for _ in range(blocks)]
        used = [b for b, u in enumerate(uses) if u]
        table = [rng.choice(used) if used and rng.random() < 0.9 else NONE for _ in range(700)]
        pairs, status = Pool(uses, table).compact()
        assert status == 0
        if pairs:
            for some in {0, 1, len(pairs) // 2, len(pairs)}:
                p = Pool(uses, table)
                p.compact(max_pairs=some)
                p.compact(work_fill=0)
                assert p.uses[:len(used)].count(0) == 0 and not any(p.uses[len(used):])


@gpu
def test_compact_with_one_hole_and_entries_that_name_nothing():
    uses = [1, 0, 2, 0, 3, 0]
    p = Pool(uses, [4, 2, 0, NONE, 6, 5, 3, 4, 0x80000000])
    assert p.compact() == ([(4, 1)], B.ST_BAD_BLOCK)
    assert p.table == [1, 2, 0, NONE, 6, 5, 3, 1, 0x80000000] and p.uses == [1, 3, 2, 0, 0, 0]
    Pool([0, 0, 1], []).compact()


# ---------------------------------------------------------------- copy

def make_planes(blocks, T, h, d, e, gap, seed=0):
    rng = np.random.default_rng(seed)
    stride = T * h * d * e + gap
    planes = [torch.from_numpy(rng.integers(0, 256, blocks * stride, dtype=np.uint8)).to(DEV) for _ in range(2)]
    pool = B.make_pool(*planes, num_blocks=blocks, block_tokens=T, num_kv_heads=h, head_dim=d, elt_bytes=e, block_stride=stride)
    return planes, pool, stride


@gpu
@pytest.mark.parametrize("T,h,d,e,gap", [(16, 8, 128, 2, 0), (16, 8, 128, 1, 48), (1, 1, 16, 1, 0), (5, 3, 16, 1, 16), (64, 5, 80, 2, 0),
                                         (7, 1, 48, 2, 32), (1, 1, 8, 4, 0), (256, 8, 128, 2, 0), (32, 1, 256, 2, 4096)])
@pytest.mark.parametrize("n", [0, 1, 2, 31])
def test_copy(T, h, d, e, gap, n):
    blocks = 70
    planes, pool, stride = make_planes(blocks, T, h, d, e, gap)
    scales = [torch.randn(blocks, h + 3, device=DEV) for _ in range(2)]
    order = np.random.default_rng(n).permutation(blocks)[:62].reshape(2, 31)
    pairs = [(int(a), int(b)) for a, b in order.T][:n]
    for with_scales in (True, False):
        for d_n in (None, n, 100):
            given = pairs + [(int(a), int(b)) for a, b in order.T][n:] if d_n == n else pairs
            status = torch.zeros(1, dtype=torch.int32, device=DEV)
            want, want_s = [p.clone() for p in planes], [s.clone() for s in scales]
            for a, b in pairs:
                for x in want:
                    x.view(blocks, stride)[b, :stride - gap] = x.view(blocks, stride)[a, :stride - gap]
                for x in want_s:
                    if with_scales:
                        x[b, :h] = x[a, :h]
            B.tutti_blocks_copy(pool, B.make_scales(*scales) if with_scales else None, words(given) if given else None,
                                None if d_n is None else words([d_n]), len(given), status)
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(planes + scales, want + want_s)) and int(status.item()) == 0


@gpu
def test_copy_skips_pairs_of_no_block():
    planes, pool, stride = make_planes(9, 16, 2, 64, 2, 0)
    for bad, bits in (((NONE, NONE), 0), ((9, 1), 1), ((1, 9), 1), ((NONE, 1), 1), ((2, NONE), 1), ((0x80000000, 0x80000001), 1)):
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        want = [p.clone() for p in planes]
        for x in want:
            x.view(9, stride)[4] = x.view(9, stride)[3]
        B.tutti_blocks_copy(pool, None, words([bad, (3, 4), bad]), None, 3, status)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(planes, want)) and int(status.item()) == bits, bad


@gpu
def test_copy_beyond_32_bits():
    """A pool of more than 4 GiB a plane: blocks at both ends of it change places."""
    blocks, stride = 4200, 1 << 20
    planes = [torch.zeros(blocks * stride, dtype=torch.uint8, device=DEV) for _ in range(2)]
    pool = B.make_pool(*planes, num_blocks=blocks, block_tokens=16, num_kv_heads=8, head_dim=128, elt_bytes=2, block_stride=stride)
    size = 16 * 8 * 128 * 2
    for i, p in enumerate(planes):
        for b in (0, 4199, 4100):
            p.view(blocks, stride)[b, :size] = torch.randint(0, 256, (size,), dtype=torch.uint8, device=DEV)
    want = [[p.view(blocks, stride)[b, :size].clone() for b in (0, 4199, 4100)] for p in planes]
    B.tutti_blocks_copy(pool, None, words([(0, 4198), (4199, 1), (4100, 4097)]), None, 3)
    torch.cuda.synchronize()
    for p, w in zip(planes, want):
        x = p.view(blocks, stride)
        assert all(torch.equal(x[b, :size], y) for b, y in zip((4198, 1, 4097), w))
        assert int(x[4198, size:].max()) == 0 and int(x[2, :size].max()) == 0


# ---------------------------------------------------------------- as they are used together

T, H, HQ, D = 16, 2, 4, 64


class Layer:
    """One layer's e4m3 cache and its calls; tables and counts are the step's."""

    def __init__(self, blocks):
        self.blocks = blocks
        self.planes = [torch.full((blocks * T * H * D,), 0x7f, dtype=torch.uint8, device=DEV) for _ in range(2)]
        self.d_scales = [torch.ones(blocks, 4, device=DEV) for _ in range(2)]
        self.pool = B.make_pool(*self.planes, num_blocks=blocks, block_tokens=T, num_kv_heads=H, head_dim=D, elt_bytes=1)
        self.scales = B.make_scales(*self.d_scales)
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)

    def step(self, qkv, seqs, table, window=0, sinks=0):
        """qkv [rows, HQ + 2H, D]; seqs (row0, n_new, n_held, table_off)."""
        rows = qkv.shape[0]
        batch = B.make_batch(words(seqs), len(seqs), max(s[1] for s in seqs), table, table.numel(), rows)
        attn = B.make_attn(HQ, B.BF16, 1.0 / math.sqrt(D), window=window)
        out = torch.empty(rows, HQ, D, dtype=torch.bfloat16, device=DEV)
        work = torch.empty(B.tutti_kv_attend_work_bytes(self.pool, batch, attn), dtype=torch.uint8, device=DEV)
        B.tutti_kv_append(self.pool, self.scales, batch, None, None, None, B.make_rows(qkv[:, HQ:HQ + H]), B.make_rows(qkv[:, HQ + H:]),
                          HQ, B.BF16, self.status)
        B.tutti_kv_attend_sinks(self.pool, self.scales, batch, attn, sinks, B.make_rows(qkv[:, :HQ]), B.make_rows(out), None, work,
                                work.numel(), self.status)
        return out

    def copy(self, pairs, n_pairs, most):
        B.tutti_blocks_copy(self.pool, self.scales, pairs, n_pairs, most, self.status)


@gpu
def test_samples_share_a_prompt_and_go_on_as_if_alone():
    """Four samples fork off a prompt, each with a copy of its open block, and go on; two end; the pool is compacted; the others go
    on.  The same sequences with blocks of their own from the start give the same bits."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(1)

    def tokens(n):
        return torch.randn(n, HQ + 2 * H, D, generator=gen, device=DEV).to(torch.bfloat16)

    blocks, width, prompt, steps = 64, 16, 77, 40
    layer = Layer(blocks)
    uses = torch.zeros(blocks, dtype=torch.int32, device=DEV)
    uses[::3] = 1                                            # blocks of others
    table = torch.full((5 * width,), -1, dtype=torch.int32, device=DEV)
    status = layer.status
    work = torch.empty(max(B.tutti_blocks_fork_work_bytes(blocks, 4), B.tutti_blocks_compact_work_bytes(blocks)), dtype=torch.uint8,
                       device=DEV)
    pairs, totals = torch.empty(64, dtype=torch.int32, device=DEV), torch.zeros(2, dtype=torch.int32, device=DEV)

    def fork(records):
        rec = np.zeros(len(records), B.FORK_DTYPE)
        for i, r in enumerate(records):
            rec[i] = (*r, (0, 0, 0))
        B.tutti_blocks_fork(uses, blocks, table, table.numel(), words(rec.view(np.uint32)), len(records), width, pairs, totals, 32, work,
                            work.numel(), status)

    # alone: a pool in which every sequence has its own blocks
    alone = Layer(4 * width)
    alone_table = words(np.random.default_rng(0).permutation(4 * width))
    x = tokens(prompt)
    fork([(0, 0, 0, 0, -(-prompt // T))])
    a = layer.step(x, [(0, prompt, prompt, 0)], table)
    b = alone.step(torch.cat([x] * 4), [(i * prompt, prompt, prompt, i * width) for i in range(4)], alone_table)
    assert all(torch.equal(a, b[i * prompt:(i + 1) * prompt]) for i in range(4))
    full = prompt // T
    fork([(0, (i + 1) * width, full, 1, 0) for i in range(4)])
    layer.copy(pairs, totals, 32)
    B.tutti_blocks_free(uses, blocks, table, table.numel(), words([(0, full + 1)]), 1, width, status)
    held, running = prompt, [0, 1, 2, 3]
    for step in range(steps):
        held += 1
        if held % T == 1:                                    # a block begins
            fork([(0, (i + 1) * width + held // T, 0, 0, 1) for i in running])
        x = tokens(len(running))
        a = layer.step(x, [(r, 1, held, (i + 1) * width) for r, i in enumerate(running)], table)
        b = alone.step(x, [(r, 1, held, i * width) for r, i in enumerate(running)], alone_table)
        assert torch.equal(a, b), step
        if step == 15:                                       # two have ended, the gaps are closed
            B.tutti_blocks_free(uses, blocks, table, table.numel(), words([(width, width), (3 * width, width)]), 2, width, status)
            running = [1, 3]
            before = int((uses != 0).sum())
            B.tutti_blocks_compact(uses, blocks, table, table.numel(), pairs, totals, 32, work, work.numel(), status)
            layer.copy(pairs, totals, 32)
            assert int((uses[:before] != 0).sum()) == before and int(uses[before:].abs().sum()) == 0 and int(totals[0]) > 0
    assert int(status.item()) == 0 == int(alone.status.item())
    B.tutti_blocks_free(uses, blocks, table, table.numel(), words([(0, 5 * width)]), 1, 5 * width, status)
    assert int(uses.sum()) == len(range(0, blocks, 3)) and bool((table == -1).all())


@gpu
def test_a_stream_outlives_its_pool():
    """600 tokens of a sequence in a pool of 8 blocks: what leaves the window is given back, new blocks come from there; the same tokens
    in a pool that holds all of them give the same bits."""
    gen = torch.Generator(device=DEV)
    gen.manual_seed(2)
    window, sinks, n = 50, 5, 600
    small, large = Layer(8), Layer(40)
    uses, table = torch.zeros(8, dtype=torch.int32, device=DEV), torch.full((40,), -1, dtype=torch.int32, device=DEV)
    work = torch.empty(B.tutti_blocks_fork_work_bytes(8, 1), dtype=torch.uint8, device=DEV)
    large_table = words(np.random.default_rng(3).permutation(40))
    for held in range(1, n + 1):
        if held % T == 1:
            gone = max(0, held - window) // T                # blocks in front of the window of place held - 1
            B.tutti_blocks_free(uses, 8, table, 40, words([(1, max(0, gone - 1))]), 1, 40, small.status)
            rec = np.zeros(1, B.FORK_DTYPE)
            rec[0] = (0, held // T, 0, 0, 1, (0, 0, 0))
            B.tutti_blocks_fork(uses, 8, table, 40, words(rec.view(np.uint32)), 1, 1, None, None, 0, work, work.numel(), small.status)
        x = torch.randn(1, HQ + 2 * H, D, generator=gen, device=DEV).to(torch.bfloat16)
        a = small.step(x, [(0, 1, held, 0)], table, window, sinks)
        b = large.step(x, [(0, 1, held, 0)], large_table, window, sinks)
        assert torch.equal(a, b) and bool(torch.isfinite(a).all()), held
    assert int(small.status.item()) == 0 == int(large.status.item())


@gpu
def test_in_a_graph_and_on_another_stream():
    """Fork, copy, free and compaction captured together: every replay does to the state what the calls do, the work memory used by
    others between."""
    rng = random.Random(5)
    uses, table, lengths = random_pool(3000, 20, 30, rng)
    records = [(i * 30, (20 + i) * 30, lengths[i] - 1, 1, 1 if lengths[i] < 30 else 0) for i in range(20)]
    planes, pool, _ = make_planes(3000, 4, 1, 16, 1, 0)
    rec = np.zeros(20, B.FORK_DTYPE)
    for i, r in enumerate(records):
        rec[i] = (*r, (0, 0, 0))
    d_rec, d_ranges = words(rec.view(np.uint32)), words([(i * 30, n) for i, n in enumerate(lengths)])
    start = [words(uses), words(table)] + [p.clone() for p in planes]
    live = [t.clone() for t in start]
    pool.k_base, pool.v_base = live[2].data_ptr(), live[3].data_ptr()
    pairs, totals = words([0] * 3000), words([0, 0])
    work = torch.empty(max(B.tutti_blocks_fork_work_bytes(3000, 20), B.tutti_blocks_compact_work_bytes(3000)), dtype=torch.uint8, device=DEV)

    def step():
        B.tutti_blocks_fork(live[0], 3000, live[1], len(table), d_rec, 20, 30, pairs, totals, 1500, work, work.numel())
        B.tutti_blocks_copy(pool, None, pairs, totals, 1500)
        B.tutti_blocks_free(live[0], 3000, live[1], len(table), d_ranges, 20, 30)
        B.tutti_blocks_compact(live[0], 3000, live[1], len(table), pairs, totals, 1500, work, work.numel())
        B.tutti_blocks_copy(pool, None, pairs, totals, 1500)

    def reset():
        for a, b in zip(live, start):
            a.copy_(b)
        torch.cuda.synchronize()

    step()
    torch.cuda.synchronize()
    want = [t.clone() for t in live]
    cpu_uses, cpu_table = list(uses), list(table)
    ref.fork(cpu_uses, cpu_table, records, 30, 1500)
    ref.free(cpu_uses, cpu_table, [(i * 30, n) for i, n in enumerate(lengths)], 30)
    ref.compact(cpu_uses, cpu_table, 1500)
    assert back(want[0]) == cpu_uses and back(want[1]) == cpu_table
    side = torch.cuda.Stream()
    reset()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(live, want))
    reset()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        reset()
        work.fill_(31 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(live, want))
        reset()
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(live, want))


# ---------------------------------------------------------------- refusals (CPU)

def code(fn, *a):
    try:
        return fn(*a, stream=0)
    except B.TuttiError as e:
        return e.code


def test_tables_are_checked():
    need = dict(fork=B.tutti_blocks_fork_work_bytes(8, 1), compact=B.tutti_blocks_compact_work_bytes(8))
    assert min(need.values()) >= 8 * 4

    def fork(uses=FAKE, blocks=8, table=FAKE, table_len=4, rec=FAKE, n=1, most=2, pairs=FAKE, n_pairs=FAKE, max_pairs=4, work=FAKE,
             size=need["fork"], status=0):
        return B.tutti_blocks_fork, uses, blocks, table, table_len, rec, n, most, pairs, n_pairs, max_pairs, work, size, status

    def free(uses=FAKE, blocks=8, table=FAKE, table_len=4, rec=FAKE, n=1, most=2, status=0):
        return B.tutti_blocks_free, uses, blocks, table, table_len, rec, n, most, status

    def compact(uses=FAKE, blocks=8, table=FAKE, table_len=4, pairs=FAKE, totals=FAKE, max_pairs=4, work=FAKE, size=need["compact"],
                status=0):
        return B.tutti_blocks_compact, uses, blocks, table, table_len, pairs, totals, max_pairs, work, size, status

    for call in (fork, free, compact):
        for bad in (dict(uses=0), dict(uses=FAKE + 4), dict(blocks=0), dict(table=0), dict(table=FAKE + 2), dict(status=FAKE + 1)):
            assert code(*call(**bad)) == B.EINVAL, (call, bad)
        assert code(*call(blocks=1 << 31)) == B.ERANGE
    for call in (fork, free):
        for bad in (dict(rec=0), dict(rec=FAKE + 4)):
            assert code(*call(**bad)) == B.EINVAL, (call, bad)
        for bad in (dict(n=B.MAX_REQ + 1), dict(most=1 << 31)):
            assert code(*call(**bad)) == B.ERANGE, (call, bad)
        assert code(*call(n=2048, most=0x7fffffff, **(dict(size=1 << 40) if call is fork else {}))) == B.ERANGE
    for call in (fork, compact):
        for bad in (dict(pairs=0), dict(pairs=FAKE + 4), dict(work=0), dict(work=FAKE + 8)):
            assert code(*call(**bad)) == B.EINVAL, (call, bad)
        assert code(*call(size=need[call.__name__] - 1)) == B.ERANGE
    assert code(*fork(n_pairs=FAKE + 2)) == B.EINVAL
    assert code(*compact(totals=0)) == code(*compact(totals=FAKE + 2)) == B.EINVAL
    assert code(*free(n=0)) == B.OK                 # nothing is enqueued
    for blocks, n in ((0, 1), (1 << 31, 1), (8, B.MAX_REQ + 1)):
        assert B.tutti_blocks_fork_work_bytes(blocks, n) == 0
    assert B.tutti_blocks_compact_work_bytes(0) == B.tutti_blocks_compact_work_bytes(1 << 31) == 0


def test_copies_are_checked():
    good = dict(num_blocks=8, block_tokens=16, num_kv_heads=2, head_dim=64, elt_bytes=2)

    def args(k=FAKE, v=FAKE, scales=None, pairs=FAKE, n_pairs=0, n=1, status=0, **kw):
        return B.make_pool(k, v, **dict(good, **kw)), scales, pairs, n_pairs, n, status

    assert code(B.tutti_blocks_copy, *args(n=0)) == B.OK
    for bad in (dict(k=0), dict(v=FAKE + 8), dict(num_blocks=0), dict(block_tokens=0), dict(num_kv_heads=0), dict(head_dim=0),
                dict(elt_bytes=0), dict(head_dim=5, num_kv_heads=1, block_tokens=1), dict(block_stride=4000), dict(block_stride=4104),
                dict(pool_layout=2), dict(block_tokens=1 << 30, num_kv_heads=64), dict(pairs=0), dict(pairs=FAKE + 4),
                dict(n_pairs=FAKE + 2), dict(status=FAKE + 2), dict(scales=B.make_scales(0, FAKE, 4)),
                dict(scales=B.make_scales(FAKE, FAKE + 2, 4)), dict(scales=B.make_scales(FAKE, FAKE, 1))):
        assert code(B.tutti_blocks_copy, *args(**bad)) == B.EINVAL, bad
    assert code(B.tutti_blocks_copy, None, *args()[1:]) == B.EINVAL


def test_the_reference_conserves_uses():
    rng = random.Random(1)
    uses, table, lengths = random_pool(400, 10, 12, rng)
    total = sum(uses)
    records = [(i * 12, (10 + i) * 12, n - 1, 1, 0) for i, n in enumerate(lengths)]
    pairs, status = ref.fork(uses, table, records, 12, 10)
    assert status == 0 and len(pairs) == 10 and sum(uses) == total + sum(lengths)
    before = sorted(u for u in uses if u)
    assert ref.compact(uses, table, 400)[1] == len(before) and sorted(uses[:len(before)]) == before
    assert ref.free(uses, table, [((10 + i) * 12, n) for i, n in enumerate(lengths)], 12) == 0 and sum(uses) == total


def test_kernels_without_scratch():
    from paper_2605_03375_amd import binding
    from test_kernel_resources import BUNDLE, _code_object, _metadata, _short_names
    with open(binding.LIB_PATH, "rb") as f:
        blob = f.read()
    found, at = {}, blob.find(BUNDLE)
    while at >= 0:
        try:
            kernels = _metadata(_code_object(blob[at:]))["amdhsa.kernels"]
            found.update(zip(_short_names([k[".name"] for k in kernels]), kernels))
        except AssertionError:      # (the bundle's name is also a string of its own)
            pass
        at = blob.find(BUNDLE, at + 1)
    blocks = {n: k for n, k in found.items() if n.startswith("k_blocks_")}
    assert len(blocks) == 9
    assert all(k[".private_segment_fixed_size"] == 0 and k[".vgpr_spill_count"] == 0 for k in blocks.values())
    # two workgroups of 1,024 threads would have 64 registers each; the others' grids count on eight of 256
    assert all(k[".vgpr_count"] <= 128 for k in blocks.values())
