"""CPU test of what the compiler gave the kernels that use a paged cache in place, read from the metadata of the built library."""
import re

from paper_2605_03375_amd import binding as B
from test_kernel_resources import BUNDLE, _code_object, _metadata, _short_names


def _kv_kernels():
    """The library holds a bundle of code objects for each of its HIP sources."""
    with open(B.LIB_PATH, "rb") as f:
        blob = f.read()
    found, at = {}, blob.find(BUNDLE)
    while at >= 0:
        try:
            kernels = _metadata(_code_object(blob[at:]))["amdhsa.kernels"]
            found.update(zip(_short_names([k[".name"] for k in kernels]), kernels))
        except AssertionError:      # (the bundle's name is also a string of its own)
            pass
        at = blob.find(BUNDLE, at + 1)
    return {n: k for n, k in found.items() if n.startswith("k_kv_")}


def test_no_scratch_and_what_a_compute_unit_holds():
    """No scratch memory; of attention kernels two workgroups fit a compute unit, which the size of its grid goes by."""
    kernels = _kv_kernels()
    families = {re.match(r"k_kv_\w+", n).group() for n in kernels}
    assert families == {"k_kv_append", "k_kv_attend", "k_kv_attend_wide", "k_kv_join"} and len(kernels) > 100
    bad = {n: (k[".private_segment_fixed_size"], k[".vgpr_spill_count"]) for n, k in kernels.items()
           if k[".private_segment_fixed_size"] or k[".vgpr_spill_count"]}
    assert not bad, bad
    for n, k in kernels.items():
        if n.startswith("k_kv_attend"):
            assert k[".vgpr_count"] <= 256 and 2 * k[".group_segment_fixed_size"] <= 160 << 10, n
