"""Attention over a window and first tokens with several KV heads side by side in a workgroup: that the rule takes each of its choices in
these cases (CPU), and each choice against 64-bit definitions (GPU)."""
import ctypes
import math
import os
import subprocess

import pytest
import torch

from paper_2605_03375_amd import binding as B
from test_kv_ops import DEV, Step
from test_kv_sinks import DTYPE, check_sinks, gpu, without_hidden

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOURCE = """
#include "attend_rules.h"
using namespace tutti;
// rows of a workgroup, its heads, wavefronts that share a head's keys; 1,000,000 where the work memory would not do
extern "C" unsigned choice_of(unsigned h, unsigned group, unsigned d, unsigned e, unsigned T, unsigned n_seq, unsigned rows, unsigned max_new,
                              unsigned window, unsigned sinks) {
  tutti_pool pool{};
  pool.num_kv_heads = h, pool.head_dim = d, pool.elt_bytes = e, pool.block_tokens = T;
  tutti_batch batch{};
  batch.n_seq = n_seq, batch.n_rows = rows, batch.max_new = max_new;
  tutti_attn attn{};
  attn.n_q_heads = h * group, attn.causal = 1, attn.window = window;
  AttendSizes s;
  if (attend_sizes(&pool, &batch, &attn, &s) != TUTTI_OK) return 0;
  const uint64_t told = s.bytes;
  const uint32_t most = most_tiles(s.rows, group, window, sinks);
  sizes_of_few(&pool, &batch, &attn, most, &s);
  return s.bytes > told ? 1000000 : s.rows * 100 + s.abreast * 10 + s.key_waves;
}
"""


def uneven(n, most, new=1):
    """n sequences of lengths between a few tokens and `most`, few long ones; every seventh has `new` new tokens, the others one."""
    held = [new + (i * 37 % n) ** 2 * (most - new) // n ** 2 for i in range(n)]
    return [(new if i % 7 == 0 else 1, held[i]) for i in range(n)]


def even(n, held, new=1):
    return [(new, held)] * n


# sequences, shape, window, first tokens; rows, heads, wavefronts a head
CASES = {
    "8x128": (even(64, 1100), dict(h=8, group=2, d=128), 1000, 4, 16, 4, 1),
    "8x128_uneven": (uneven(60, 1900), dict(h=8, group=1, d=128, gap=16), 1000, 40, 16, 4, 1),
    "8x128_drafts": (uneven(64, 1400, 5), dict(h=8, group=4, d=128), 800, 70, 32, 4, 1),
    "4x112_head_major_12": (uneven(64, 2300, 3), dict(h=4, group=2, d=112, T=12, hnd=True), 1700, 4, 16, 4, 1),
    "4x64_drafts_10": (uneven(63, 2600, 6), dict(h=4, group=3, d=64, T=10, dtype="fp16"), 1700, 129, 32, 4, 1),
    "5x80": (uneven(64, 2900), dict(h=5, group=1, d=80, T=32), 2600, 4, 16, 5, 1),
    "5x80_drafts_10": (uneven(64, 3300, 8), dict(h=5, group=4, d=80, T=10, dtype="fp16"), 2600, 33, 32, 5, 1),
    "5x128_head_major": (uneven(64, 3300), dict(h=5, group=4, d=128, hnd=True), 2600, 4, 16, 5, 1),
    "3x96": (uneven(64, 5400), dict(h=3, group=2, d=96), 4400, 16, 16, 3, 1),
    "3x128_drafts_head_major_24": (uneven(64, 5000, 4), dict(h=3, group=8, d=128, T=24, hnd=True), 4400, 300, 32, 3, 1),
    "2x64": (even(64, 3600), dict(h=2, group=4, d=64), 3300, 4, 16, 2, 2),
    "2x128_uneven": (uneven(64, 4400), dict(h=2, group=8, d=128, gap=32, dtype="fp16"), 3300, 100, 16, 2, 2),
    "2x48_drafts_head_major_12": (uneven(64, 4400, 7), dict(h=2, group=3, d=48, T=12, hnd=True), 3300, 4, 32, 2, 2),
    "8x128_two_of_few": (even(100, 300), dict(h=8, group=2, d=128), 90, 20, 16, 2, 2),
    "8x64_two_of_few_10": (uneven(120, 600, 5), dict(h=8, group=4, d=64, T=10), 300, 4, 32, 2, 2),
    "4x80_one_of_few_head_major": (uneven(60, 900, 9), dict(h=4, group=2, d=80, hnd=True), 300, 4, 32, 1, 4),
    "5x64_420": (uneven(420, 200), dict(h=5, group=2, d=64), 70, 7, 16, 5, 1),
    "3x128_700_12": (uneven(700, 120), dict(h=3, group=1, d=128, T=12, hnd=True), 50, 3, 16, 3, 1),
    "8x128_130_drafts": (uneven(130, 700, 5), dict(h=8, group=4, d=128), 500, 4, 32, 4, 1),
    "2x64_150_long": (uneven(150, 2100), dict(h=2, group=4, d=64), 1700, 60, 16, 2, 2),
}


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    d = tmp_path_factory.mktemp("attend_rules")
    src, lib = d / "rules.cpp", d / "rules.so"
    src.write_text(SOURCE)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", f"-I{ROOT}/paper_2605_03375_amd/csrc",
                    f"-I{ROOT}/include", str(src), "-o", str(lib)], check=True)
    return ctypes.CDLL(str(lib))


@pytest.mark.parametrize("name", CASES)
def test_the_rule_takes_this_choice(rules, name):
    seqs, shape, window, sinks, rows, heads, waves = CASES[name]
    for e in (1, 2):
        got = rules.choice_of(shape["h"], shape["group"], shape["d"], e, shape.get("T", 16), len(seqs), sum(s[0] for s in seqs),
                              max(s[0] for s in seqs), window, sinks)
        assert got == rows * 100 + heads * 10 + waves


def test_every_choice_is_among_the_cases():
    """Workgroups of one to five heads, for 16 and 32 rows, up to 64 sequences and more; blocks that 16 divides or not; both layouts."""
    there = {(rows, heads) for *_, rows, heads, _ in CASES.values()}
    assert there >= {(16, n) for n in (2, 3, 4, 5)} | {(32, n) for n in (1, 2, 3, 4, 5)}      # (16, 1) is what test_kv_sinks has
    assert {(heads, len(seqs) > 64) for seqs, *_, heads, _ in CASES.values()} >= {(n, more) for n in (2, 3, 4, 5) for more in (False, True)}
    for n in (2, 3, 4, 5):
        shapes = [c[1] for c in CASES.values() if c[5] == n]
        assert {s.get("T", 16) % 16 == 0 for s in shapes} == {s.get("hnd", False) for s in shapes} == {False, True}


def test_work_memory_is_what_the_caller_was_told(rules):
    for h in (1, 2, 3, 4, 5, 6, 7, 8, 12, 20):
        for n in (1, 3, 64, 65, 130, 513, 2048):
            for window in (1, 60, 1000, 5000, 100000, 0xffffffff):
                for new, group in ((1, 1), (5, 4), (40, 8)):
                    for sinks in (1, 100, 0x7fffffff):
                        assert 0 < rules.choice_of(h, group, 128, 2, 16, n, n * new, new, window, sinks) < 1000000


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("name", CASES)
def test_heads_side_by_side(name, cache):
    seqs, shape, window, sinks, *_ = CASES[name]
    st = Step(seqs, cache="e4m3" if cache == "e4m3" else None, seed=len(seqs) + window, **shape)
    without_hidden(st, window, sinks)
    check_sinks(st, window, sinks)


def tiles_a_part(st, window, sinks):
    """What the kernel put in front of its work memory: key tiles of 32 that a part has."""
    out = torch.empty(st.rows, st.hq, st.d, dtype=st.d_q.dtype, device=DEV)
    attn = B.make_attn(st.hq, DTYPE[st.dtype], 1.0 / math.sqrt(st.d), window=window)
    work = torch.empty(B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn) // 4, dtype=torch.int32, device=DEV)
    B.tutti_kv_attend_sinks(st.pool, st.scales, st.batch, attn, sinks, B.make_rows(st.d_q), B.make_rows(out), None, work, work.numel() * 4)
    return int(work[0].item())


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("seqs,shape,window", [
    ([(700, 2600)], dict(h=4, group=4, d=64), 1500),                                     # tiles of 128 rows
    (uneven(40, 3000, 1) + even(36, 2900, 8), dict(h=8, group=4, d=64), 2600)])          # of 32, more than 64 sequences
def test_more_joined_rows_than_a_grid_takes_at_once(seqs, shape, window, cache):
    """More than 8,192 rows of sequences that are split: the join goes round again."""
    st = Step(seqs, cache="e4m3" if cache == "e4m3" else None, seed=9, **shape)
    without_hidden(st, window, 10)
    check_sinks(st, window, 10)
    a_part = tiles_a_part(st, window, 10)
    seen = [min(held, window + 7) // 32 for _, held in seqs]
    assert sum(new * st.hq for (new, _), n in zip(seqs, seen) if n > a_part) > 8192, a_part
