"""How the attention kernels that keep keys and values in LDS order their reads of it and what fills it: the built kernels (CPU), and
calls that repeat to the bit."""
import re
import subprocess

import pytest

from paper_2605_03375_amd import binding as B
from test_kernel_resources import BUNDLE, _code_object, _short_names
from test_kv_ops import Step, check_attend, run_attend, same

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
LINE = re.compile(r"\t(\S+)[^/]*// ([0-9A-F]+):[^<]*(?:<[^>+]+(?:\+0x([0-9a-f]+))?>)?")


def _listing(tmp_path):
    """{kernel: its instructions in order, (name, offset, offset that it may branch to)} of the wide attention kernels."""
    with open(B.LIB_PATH, "rb") as f:
        blob = f.read()
    found, at = {}, blob.find(BUNDLE)
    while at >= 0:
        try:
            code = _code_object(blob[at:])
        except AssertionError:      # (the bundle's name is also a string of its own)
            code = b""
        if b"k_kv_attend_wide" in code:
            path = tmp_path / "kernels.co"
            path.write_bytes(code)
            text = subprocess.run([OBJDUMP, "-d", "--mcpu=gfx950", str(path)], capture_output=True, text=True, check=True).stdout
            for part in re.split(r"\n(?=[0-9a-f]{16} <)", text):
                head = re.match(r"([0-9a-f]{16}) <([^>]*k_kv_attend_wide[^>]*)>:", part)
                if head:
                    begin = int(head[1], 16)
                    found[head[2]] = [(m[1], int(m[2], 16) - begin, int(m[3] or "0", 16) if "branch" in m[1] else None)
                                      for m in map(LINE.match, part.split("\n")) if m]
        at = blob.find(BUNDLE, at + 1)
    return dict(zip(_short_names(list(found)), found.values()))


def loads_that_overtake(code):
    """Offsets of loads into LDS that some path reaches from a read of LDS without a barrier between them."""
    index = {offset: i for i, (_, offset, _) in enumerate(code)}
    todo, seen, found = [i for i, (name, _, _) in enumerate(code) if name.startswith("ds_read")], set(), []
    while todo:
        i = todo.pop()
        name, offset, target = code[i]
        if i in seen or name == "s_barrier":
            continue
        seen.add(i)
        if name.startswith("global_load_lds"):
            found.append(offset)
        if target is not None:
            todo.append(index[target])
        if name not in ("s_branch", "s_endpgm"):
            todo.append(i + 1)
    return sorted(found)


def test_the_search():
    straight = [("ds_read_b128", 0, None), ("s_barrier", 8, None), ("global_load_lds_dwordx4", 12, None), ("s_endpgm", 20, None)]
    assert loads_that_overtake(straight) == []
    # the barrier is in a loop's turns but the first
    around = [("ds_read_b128", 0, None), ("s_branch", 8, 16), ("s_barrier", 12, None), ("global_load_lds_dwordx4", 16, None),
              ("s_cbranch_scc1", 24, 12), ("s_endpgm", 28, None)]
    assert loads_that_overtake(around) == [16]


def test_no_plane_of_lds_is_filled_while_it_may_be_read(tmp_path):
    """A wavefront that asks for rows straight into LDS has met the others since it last read LDS: what it overwrites nobody reads any
    more.  (Kernels of 16-bit blocks; those of e4m3 blocks are the same source, but fill by stores that may follow reads of other
    planes.)"""
    direct = {n: c for n, c in _listing(tmp_path).items() if any(name.startswith("global_load_lds") for name, _, _ in c)}
    assert len(direct) >= 20 and all(re.match(r"k_kv_attend_wide<\w+, false,", n) for n in direct)
    for code in direct.values():
        assert {"s_barrier", "ds_read_b128", "ds_read_b64_tr_b16"} <= {name for name, _, _ in code}
    bad = {n: [hex(x) for x in loads_that_overtake(c)] for n, c in direct.items()}
    assert not any(bad.values()), {n: x for n, x in bad.items() if x}


@pytest.mark.gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("n_new,window", [(20, 0), (24, 0), (49, 0), (200, 0), (200, 70)])
def test_wide_twice_the_same(n_new, window, T, cache):
    """Tiles in which some wavefronts have no rows, or see nothing of a part's first keys, and so reach its first turn before others."""
    st = Step([(n_new, 1500), (1, 900)], T=T, group=2, d=128, cache="e4m3" if cache == "e4m3" else None, seed=n_new + window)
    out, lse = check_attend(st, window=window)
    for fill in (0x00, 0x7f, 0x3c, 0xff):
        again = run_attend(st, window=window, work_fill=fill)
        assert same(out, again[0]) and same(lse, again[1])
