"""Attention at the ends of the types' ranges, on the GPU against 64 bits: scores, weights and values that are very large or very small."""
import numpy as np
import pytest

import kv_reference as ref
from test_kv_ops import Step, run_attend

gpu = pytest.mark.gpu
STEPS = [[(1, 50)], [(1, 3000)], [(5, 40)], [(40, 60)], [(40, 2500)]]     # one tile and split, few and many rows


def by_name(s):
    return "-".join(f"{a}of{b}" for a, b in s)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("seqs", STEPS, ids=by_name)
def test_scores_far_below_zero(seqs, T, cache):
    """Every key's score is -2^126 (a quarter of what 32 bits hold; times log2(e) -1.2e38): they share the weight evenly, however low."""
    st = Step(seqs, T=T, cache="e4m3" if cache == "e4m3" else None)
    big = 2.0 ** 60
    st.q[:] = big
    st.cpu.planes[0][:] = ref.to_e4m3(-1.0) if cache == "e4m3" else -big
    if cache == "e4m3":
        st.cpu.scales[0][:] = big
        st.cpu.scales[1][:] = 1.0        # (their logarithms would be lost beside such scores)
    out, lse, status = run_attend(st.to_gpu(), sm_scale=1.0)
    assert status == 0
    for (row0, n_new, n_held, off) in st.seqs:
        places = np.arange(n_held)
        blocks = st.table[off + places // T]
        v = st.cpu.planes[1][blocks, places % T]
        if cache == "e4m3":
            v = ref.E4M3[v] * st.cpu.scales[1][blocks][:, :, None]
        for i in range(n_new):
            n = n_held - n_new + i + 1
            # all weights are one value: the products and sums in 32 bits, the result's rounding; e4m3: powers of two of the scales
            # times reciprocals and logarithms to 2^-21
            want = np.repeat(v[:n].astype(np.float64).mean(0), st.group, 0)
            slack = np.repeat(np.abs(v[:n]).astype(np.float64).mean(0), st.group, 0) * ((n / 8 + 64) * ref.F32 + 2.0 ** -20)
            assert (np.abs(out[row0 + i] - want) <= 1.01 * ref.UNIT[st.dtype] * np.abs(want) + slack).all(), i
            assert (np.abs(lse[row0 + i] + 2.0 ** 126) <= 2.0 ** (126 - 20)).all(), i
