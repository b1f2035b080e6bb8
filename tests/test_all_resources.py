"""CPU test of what the compiler gave every kernel of the built library, one bundle of code objects for each of its HIP sources."""
import re

from test_kernel_resources import BUNDLE, _code_object, _metadata, _short_names
from paper_2605_03375_amd import binding as B


def all_kernels(blob):
    found, at = {}, blob.find(BUNDLE)
    while at >= 0:
        try:
            kernels = _metadata(_code_object(blob[at:]))["amdhsa.kernels"]
            found.update(zip(_short_names([k[".name"] for k in kernels]), kernels))
        except AssertionError:      # (the bundle's name is also a string of its own)
            pass
        at = blob.find(BUNDLE, at + 1)
    return found


def test_no_kernel_of_any_source_uses_scratch():
    """Attention has kernels with and without first tokens, in sources of their own; the widest of them are close to all registers."""
    with open(B.LIB_PATH, "rb") as f:
        found = all_kernels(f.read())
    number = {}
    for n in found:
        family = re.match(r"\w+", n).group()
        kind = (family, n.rstrip(">").split(", ")[-1]) if family in ("k_kv_attend", "k_kv_attend_wide", "k_kv_join") else (family, "")
        number[kind] = number.get(kind, 0) + 1
    for sinks in ("true", "false"):
        assert number["k_kv_attend", sinks] == 64 and number["k_kv_attend_wide", sinks] == 48 and number["k_kv_join", sinks] == 48, number
    assert {f for f, _ in number} >= {"k_layer", "k_move", "k_kv_append", "k_blocks_fork", "k_blocks_move", "k_blocks_copy"} and len(found) > 550
    bad = {n: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for n, k in found.items()
           if k[".private_segment_fixed_size"] or k[".vgpr_spill_count"]}
    assert not bad, f"scratch bytes a lane, spilled vector registers: {bad}"


def test_workgroups_that_the_grids_of_blocks_count_on():
    """Compaction's last launch has 2,048 workgroups of 256 threads, eight a compute unit, which have 64 registers a thread; a fork in one
    launch is one workgroup of 1,024 threads, which has 128."""
    with open(B.LIB_PATH, "rb") as f:
        found = all_kernels(f.read())
    assert found["k_blocks_move"][".vgpr_count"] <= 64 and found["k_blocks_fork_small"][".vgpr_count"] <= 128
