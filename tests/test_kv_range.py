"""Attention at the ends of the types' ranges, on the GPU against 64 bits: scores, weights and values that are very large or very small."""
import math

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


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("size", [16, 26, 30, 34, 60, 110])
@pytest.mark.parametrize("seqs", STEPS, ids=by_name)
def test_scores_of_any_size(seqs, size, T, cache):
    """Products of whole numbers times 2^size, exact in 32 bits, by a factor that is not: all weight is with the largest, in equal shares,
    whatever the rounding of the factor's product is beside 1."""
    st = Step(seqs, T=T, cache="e4m3" if cache == "e4m3" else None)
    rng = np.random.default_rng(size)
    st.q = rng.integers(-2, 3, st.q.shape).astype(np.float32)
    k = rng.integers(-2, 3, st.cpu.planes[0].shape).astype(np.float32)
    q, products = st.q.astype(np.float64), k.astype(np.float64)
    st.q = st.q * np.float32(2.0 ** (size - size // 2))
    if cache == "e4m3":
        st.cpu.planes[0], st.cpu.scales[0][:], st.cpu.scales[1][:] = ref.to_e4m3(k), 2.0 ** (size // 2), 1.0
    else:
        st.cpu.planes[0] = k * np.float32(2.0 ** (size // 2))
    out, lse, status = run_attend(st.to_gpu(), sm_scale=1.0 / 3)
    assert status == 0
    scale = float(np.float32(1.0 / 3)) * 2.0 ** size
    for (row0, n_new, n_held, off) in st.seqs:
        places = np.arange(n_held)
        blocks = st.table[off + places // T]
        v, kk = st.cpu.planes[1][blocks, places % T], products[blocks, places % T]
        if cache == "e4m3":
            v = ref.E4M3[v]
        for i in range(n_new):
            for head in range(st.hq):
                n = n_held - n_new + i + 1
                s = kk[:n, head // st.group] @ q[row0 + i, head]
                top = v[:n, head // st.group][s == s.max()].astype(np.float64)
                want, size_of = top.mean(0), np.abs(top).mean(0)
                slack = size_of * (1.01 * ref.UNIT[st.dtype] + (n / 8 + 64) * ref.F32 + 2.0 ** -20)
                assert (np.abs(out[row0 + i, head] - want) <= slack).all(), (i, head)
                assert abs(lse[row0 + i, head] - scale * s.max()) <= 2.0 ** -20 * abs(scale * s.max()) + 8, (i, head)


@gpu
@pytest.mark.parametrize("dtype,cache", [("bf16", None), ("fp16", None), ("bf16", "e4m3"), ("fp16", "e4m3")])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("above", [10, 20, 25.5, 30])
@pytest.mark.parametrize("n_new,n_seq", [(1, 1), (40, 1), (1, 600)])
def test_many_small_weights(n_new, n_seq, above, T, dtype, cache):
    """One key whose weight is 2^above times that of each other one, and whose value is 0: what the others add up to is the result.  A
    weight keeps its type's precision down to 2^-21 of the largest, and is off by 2^-32 of that at most below.  (600 sequences, of the same
    blocks, are not split.)"""
    st = Step([(n_new, 8000)], T=T, dtype=dtype, cache=cache, h=1, group=1)
    if n_seq > 1:
        st.seqs, st.rows = [(i, 1, 8000, 0) for i in range(n_seq)], n_seq
        st.q, st.k, st.v = (np.zeros((n_seq, 1, st.d), np.float32) for _ in range(3))
    sm_scale = above * math.log(2.0)
    st.q[:] = 0
    st.q[:, :, 0] = 1
    k, v = st.cpu.planes
    rng = np.random.default_rng(4)
    codes = rng.uniform(0.5, 1.0, v.shape)
    v[:], k[:] = (ref.to_e4m3(codes), 0) if cache else (ref.round16(codes, dtype), 0)
    for s in st.cpu.scales:
        s[:] = 1.0
    first = st.table[0]
    k[first, 3, 0, 0] = ref.to_e4m3(1.0) if cache else 1.0
    v[first, 3] = 0
    out, lse, status = run_attend(st.to_gpu(), sm_scale=sm_scale)
    assert status == 0
    places = np.arange(8000)
    values = v[st.table[places // T], places % T, 0]
    values = ref.E4M3[values] if cache else values.astype(np.float64)
    u_w = ref.UNIT["fp16" if cache else dtype]
    for i in range(st.rows):
        n = 8000 - n_new + i + 1 if n_seq == 1 else 8000
        w = 2.0 ** (above * (places[:n] == 3) - above)
        want = w @ values[:n] / w.sum()
        ds = (st.d + 8) * ref.F32 * sm_scale + 2.0 ** -21
        slack = (1.01 * ref.UNIT[dtype] + u_w + 2 * ds + 2 * (n / 8 + 64) * ref.F32) * want + n * 2.0 ** -32 + 2.0 ** -25
        assert (np.abs(out[i, 0] - want) <= slack).all(), (i, np.abs(out[i, 0] - want).max(), slack.min())
        assert abs(lse[i, 0] - (sm_scale + math.log(w.sum()))) <= ds + (n / 8 + 64) * ref.F32 + 2.0 ** -18


@gpu
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("seqs", [[(1, 900)], [(30, 300)], [(200, 700)]], ids=by_name)
def test_largest_values(seqs, T):
    """Values that are all the largest of fp16: so is every result, and it does not overflow by the roundings of its weights."""
    st = Step(seqs, T=T, dtype="fp16", spread=2.0)
    st.cpu.planes[1][:] = 65504.0
    st.cpu.planes[1][:, :, 1] = -65504.0
    out, _, status = run_attend(st.to_gpu())
    assert status == 0
    want = np.where(np.arange(st.hq) < st.group, 65504.0, -65504.0)[None, :, None]
    assert (np.abs(out - want) <= 65504.0 * (2 * ref.UNIT["fp16"] + (seqs[0][1] / 8 + 64) * ref.F32)).all()


@gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T", [16, 24])
@pytest.mark.parametrize("n_new", [4, 60, 150])
def test_infinite_values(n_new, T, dtype):
    """Infinities of both signs and NaN, in tiles that all rows see and in tiles that some do: each column is what the values that a row
    sees add up to."""
    n_held, marks = n_new + 400, {}
    for at in (5, 333, 400, 402):
        marks[at] = [(1, math.inf), (2, -math.inf), (3, math.nan)]
    marks[7], marks[401], marks[403] = [(4, math.inf)], [(4, -math.inf), (5, math.inf)], [(5, -math.inf), (6, -math.inf)]
    st = Step([(n_new, n_held)], T=T, dtype=dtype, d=128)
    for at, columns in marks.items():
        for column, x in columns:
            st.cpu.planes[1][st.table[at // T], at % T, 1, column] = x
    out, lse, status = run_attend(st.to_gpu())
    assert status == 0 and np.isfinite(lse).all()
    for i in range(n_new):
        want = np.zeros(st.d)
        for at, columns in marks.items():
            if at <= n_held - n_new + i:
                for column, x in columns:
                    with np.errstate(invalid="ignore"):
                        want[column] += x
        for head in range(st.hq):
            got = np.where(np.isfinite(out[i, head]), 0.0, out[i, head])
            assert np.array_equal(got, want if head // st.group == 1 else np.zeros(st.d), equal_nan=True), (i, head)


@gpu
@pytest.mark.parametrize("dtype,cache", [("bf16", None), ("fp16", None), ("fp16", "e4m3")])
@pytest.mark.parametrize("seqs,T", [([(1, 512)], 16), ([(3, 300), (1, 77)], 16), ([(7, 90)], 24)], ids=str)
def test_weights_of_few_queries_add_no_rounding(seqs, T, dtype, cache):
    """Two numbers to a weight: what is left of its rounding is that of the second, and the result's own is all that shows."""
    st = Step(seqs, T=T, dtype=dtype, cache=cache, spread=2.0)
    out, _, status = run_attend(st.to_gpu())
    assert status == 0
    for (row0, n_new, n_held, off) in st.seqs:
        places = np.arange(n_held)
        blocks = st.table[off + places // T]
        k, v = (p[blocks, places % T] for p in st.cpu.planes)
        if cache:
            k, v = (ref.E4M3[x] * s[blocks][:, :, None] for x, s in zip((k, v), st.cpu.scales))
        k, v = k.astype(np.float64), v.astype(np.float64)
        for i in range(n_new):
            for head in range(st.hq):
                n, kv = n_held - n_new + i + 1, head // st.group
                q = st.q[row0 + i, head].astype(np.float64)
                s = k[:n, kv] @ q / math.sqrt(st.d)
                w = np.exp(s - s.max())
                w /= w.sum()
                want, mag = w @ v[:n, kv], w @ np.abs(v[:n, kv])
                size = (np.abs(k[:n, kv]) @ np.abs(q)).max() / math.sqrt(st.d)
                ds = (st.d + 8) * ref.F32 * size + 2 * ref.F32 * np.abs(s).max() + 2.0 ** -21
                bound = (2.0 * ref.UNIT[dtype] ** 2 + 2 * ds + 2 * (n / 8 + 64) * ref.F32) * mag * 1.01 + \
                    ref.UNIT[dtype] * np.abs(want) * 1.01 + 2.0 ** -25
                assert (np.abs(out[row0 + i, head] - want) <= bound).all(), (i, head)
