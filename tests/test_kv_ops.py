"""The calls that use a paged cache in place, tutti_kv_append and tutti_kv_attend: against 64-bit definitions on the GPU, and
what they refuse (CPU)."""
import math

import numpy as np
import pytest
import torch

import kv_reference as ref
from paper_2605_03375_amd import binding as B

DEV = "cuda:0"
FAKE = 0x10000
gpu = pytest.mark.gpu


# ---------------------------------------------------------------- a step on the GPU and the same on the CPU

class Step:
    """A pool with some sequences' tokens in it and NaN everywhere else, on both sides, and a step's queries, keys, values."""

    def __init__(self, seqs, *, T=16, h=2, group=2, d=64, dtype="bf16", cache=None, hnd=False, seed=0, gap=0, extra_blocks=3,
                 spread=1.0, pad_rows=0, held_before=True):
        rng = np.random.default_rng(seed)
        self.T, self.h, self.group, self.d, self.dtype, self.hnd = T, h, group, d, dtype, hnd
        self.hq, self.kind = h * group, cache or dtype
        self.rng = rng
        need = [-(-n_held // T) for _, n_held in seqs]
        self.blocks = sum(need) + extra_blocks
        order = rng.permutation(self.blocks)
        self.table = np.concatenate([order[:sum(need)], [0]]).astype(np.uint32)[:sum(need)]
        self.seqs, row, off = [], pad_rows, 0
        for (n_new, n_held), n in zip(seqs, need):
            self.seqs.append((row, n_new, n_held, off))
            row, off = row + n_new + pad_rows, off + n
        self.rows = row
        self.cpu = ref.Cache(self.blocks, T, h, d, self.kind)
        for plane, scales in zip(self.cpu.planes, self.cpu.scales):
            if self.kind == "e4m3":
                plane[:] = 0x7f
                scales[:] = np.nan
            else:
                plane[:] = np.nan
            for _, n_new, n_held, off in self.seqs:
                upto = n_held if held_before else n_held - n_new
                for n in range(-(-upto // T)):
                    some = min(T, upto - n * T)
                    x = rng.standard_normal((some, h, d)) * spread * np.exp(0.5 * rng.standard_normal((1, h, 1)))
                    b = self.table[off + n]
                    if self.kind == "e4m3":
                        for head in range(h):
                            scales[b, head] = ref.scale_for(x[:, head])
                            plane[b, :some, head] = ref.to_e4m3(x[:, head] / scales[b, head])
                    else:
                        plane[b, :some] = ref.round16(x, self.kind)
        self.q, self.k, self.v = (ref.round16(rng.standard_normal((max(1, self.rows), n, d)) * spread, dtype)
                                  for n in (self.hq, h, h))
        self.gap = gap

    def to_gpu(self):
        """Planes in the pool's layout (with `gap` bytes behind each block), scales, records; NaN in all gaps."""
        T, h, d = self.T, self.h, self.d
        e = 1 if self.kind == "e4m3" else 2
        self.stride = T * h * d * e + self.gap
        self.d_planes, self.d_scales = [], []
        for plane, scales in zip(self.cpu.planes, self.cpu.scales):
            x = plane.transpose(0, 2, 1, 3) if self.hnd else plane
            x = np.ascontiguousarray(x).reshape(self.blocks, -1)
            if e == 1:
                raw = torch.from_numpy(x.copy())
            else:
                raw = torch.from_numpy(x).to(ref.TYPES[self.kind]).view(torch.uint8).reshape(self.blocks, -1)
            padded = torch.full((self.blocks, self.stride), 0x7f, dtype=torch.uint8)
            padded[:, :raw.shape[1]] = raw
            self.d_planes.append(padded.to(DEV))
            s = torch.full((self.blocks, -(-h // 4) * 4 + 4), math.nan)
            s[:, :h] = torch.from_numpy(scales)
            self.d_scales.append(s.to(DEV))
        self.pool = B.make_pool(*self.d_planes, num_blocks=self.blocks, block_tokens=T, num_kv_heads=h, head_dim=d, elt_bytes=e,
                                block_stride=self.stride, pool_layout=B.LAYOUT_HND if self.hnd else B.LAYOUT_NHD)
        self.scales = B.make_scales(*self.d_scales) if e == 1 else None
        self.set_batch()
        t = ref.TYPES[self.dtype]
        # queries, keys and values beside each other in one row, and 16 bytes behind it
        n = (self.hq + 2 * h) * d
        self.d_qkv = torch.full((max(1, self.rows), n + 8), math.nan, dtype=t, device=DEV)
        for at, x in ((0, self.q), (self.hq * d, self.k), ((self.hq + h) * d, self.v)):
            self.d_qkv[:, at:at + x.shape[1] * d] = torch.from_numpy(x.reshape(x.shape[0], -1)).to(t).to(DEV)
        part = [self.d_qkv[:, a:b].unflatten(1, (-1, d)) for a, b in ((0, self.hq * d), (self.hq * d, (self.hq + h) * d),
                                                                     ((self.hq + h) * d, n))]
        self.d_q, self.d_k, self.d_v = part
        self.status = torch.zeros(1, dtype=torch.int32, device=DEV)
        return self

    def set_batch(self, max_new=None, n_rows=None, table_len=None):
        rec = np.array(self.seqs, np.uint32).reshape(-1, 4)
        self.d_seqs = torch.from_numpy(rec.view(np.int32).copy()).to(DEV)
        self.d_table = torch.from_numpy(self.table.view(np.int32).copy()).to(DEV)
        self.batch = B.make_batch(self.d_seqs, len(self.seqs), max([s[1] for s in self.seqs] + [1]) if max_new is None else max_new,
                                  self.d_table, len(self.table) if table_len is None else table_len,
                                  self.rows if n_rows is None else n_rows)

    def cache_back(self):
        """Planes as on the CPU, the bytes behind the blocks, and the scales."""
        T, h, d = self.T, self.h, self.d
        e = 1 if self.kind == "e4m3" else 2
        got = []
        for plane in self.d_planes:
            raw = plane.cpu()
            assert bool((raw[:, T * h * d * e:] == 0x7f).all()), "bytes behind a block were written"
            x = raw[:, :T * h * d * e].contiguous()
            x = x.numpy() if e == 1 else x.view(ref.TYPES[self.kind]).float().numpy()
            x = x.reshape(self.blocks, *((h, T) if self.hnd else (T, h)), d)
            got.append(x.transpose(0, 2, 1, 3) if self.hnd else x)
        return got, [s.cpu().numpy()[:, :h] for s in self.d_scales]


def same(a, b):
    return np.array_equal(a, b, equal_nan=a.dtype.kind == "f")


def same_codes(a, b):
    """Codes alike, but for which of the two NaN codes it is."""
    return np.array_equal(np.where(a & 0x7f == 0x7f, 0x7f, a), np.where(b & 0x7f == 0x7f, 0x7f, b))


def make_angles(n_pos, rot, seed=0):
    half = rot // 2
    angle = np.arange(n_pos)[:, None] * 10000.0 ** (-np.arange(half) / half)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


# ---------------------------------------------------------------- append

def run_append(st, rope=None, in_place=False, with_q=True, max_new=None):
    st.to_gpu()
    if max_new is not None:
        st.set_batch(max_new=max_new)
    t = ref.TYPES[st.dtype]
    q_out = st.d_q if in_place else torch.full((max(1, st.rows), st.hq, st.d), math.nan, dtype=t, device=DEV)
    r = None
    if rope is not None:
        st.d_cos = torch.from_numpy(rope["cos_sin"]).to(DEV)
        pos = None if rope["pos"] is None else torch.from_numpy(rope["pos"].astype(np.int32)).to(DEV)
        r = B.make_rope(st.d_cos, rope["rot"], d_pos=pos, pairs=rope["pairs"], interleaved=rope["interleaved"])
    rows = [B.make_rows(x) for x in (st.d_q, q_out, st.d_k, st.d_v)]
    if not with_q:
        rows[0] = rows[1] = None
    B.tutti_kv_append(st.pool, st.scales, st.batch, r, *rows, st.hq, {"bf16": B.BF16, "fp16": B.FP16}[st.dtype], st.status)
    torch.cuda.synchronize()
    return q_out.float().cpu().numpy(), int(st.status.item())


def check_append(st, rope=None, table_len=None, **kw):
    q_out, status = run_append(st, rope, **kw)
    want_q, want_status = ref.append(st.cpu, st.dtype, st.seqs, st.table, st.q, st.k, st.v, rope, table_len)
    assert status == want_status
    planes, scales = st.cache_back()
    if st.kind == "e4m3":
        assert all(same(a, b) for a, b in zip(scales, st.cpu.scales))
        assert all(same_codes(a, b) for a, b in zip(planes, st.cpu.planes))
    else:
        assert all(same(a, b) for a, b in zip(planes, st.cpu.planes))
    if kw.get("with_q", True):
        if kw.get("in_place"):
            want_q = np.where(np.isnan(want_q), st.q, want_q)
        assert same(q_out, want_q)
    return status


SHAPES = [  # (new, held) of each sequence
    [(1, 1)], [(1, 16)], [(1, 17)], [(1, 4100)], [(3, 3)], [(16, 16)], [(17, 33)], [(40, 75)], [(1, 5), (1, 16), (1, 32), (1, 33)],
    [(0, 0), (1, 9), (0, 50), (70, 71), (2, 18)], [(1, 20 + 3 * i) for i in range(70)], [(129, 200), (64, 64), (5, 500)]]


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("seqs", SHAPES, ids=lambda s: f"{len(s)}seq_{sum(a for a, _ in s)}")
def test_append_lengths(seqs, cache):
    rope = dict(cos_sin=make_angles(4200, 64), rot=64, interleaved=False, pos=None, pairs=None)
    st = Step(seqs, cache="e4m3" if cache == "e4m3" else None, held_before=False, seed=len(seqs))
    assert check_append(st, rope) == 0


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T,h,group,d,rot,interleaved,hnd,dtype,gap", [
    (16, 8, 4, 128, 128, False, False, "bf16", 0), (16, 8, 4, 128, 128, True, True, "fp16", 0), (32, 1, 8, 128, 64, False, True, "bf16", 48),
    (64, 5, 1, 80, 80, False, False, "bf16", 0), (64, 2, 1, 80, 40, False, True, "fp16", 16), (16, 3, 2, 112, 56, True, False, "bf16", 0),
    (1, 2, 3, 16, 2, False, False, "fp16", 0), (5, 4, 1, 96, 48, False, True, "bf16", 16), (48, 2, 2, 64, 62, True, False, "bf16", 0),
    (8, 1, 1, 32, 32, False, False, "fp16", 32), (128, 1, 2, 64, 6, False, False, "bf16", 0)])
def test_append_layouts(cache, T, h, group, d, rot, interleaved, hnd, dtype, gap):
    rope = dict(cos_sin=make_angles(600, rot), rot=rot, interleaved=interleaved, pos=None, pairs=None)
    st = Step([(1, 7), (100, 300), (1, 130), (9, 9)], T=T, h=h, group=group, d=d, dtype=dtype, hnd=hnd, gap=gap, pad_rows=2,
              cache="e4m3" if cache == "e4m3" else None, held_before=False, seed=T + d)
    assert check_append(st, rope) == 0


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("pairs", [[16, 24, 24], [11, 30, 23], [0, 64], [1, 0, 2, 61]])
@pytest.mark.parametrize("interleaved", [False, True])
def test_append_axes(pairs, interleaved, cache):
    seqs = [(50, 90), (7, 7), (1, 33)]
    st = Step(seqs, h=2, d=128, cache="e4m3" if cache == "e4m3" else None, held_before=False, seed=sum(pairs[:1]))
    pos = np.random.default_rng(5).integers(0, 200, (len(pairs), st.rows))
    rope = dict(cos_sin=make_angles(200, 128), rot=128, interleaved=interleaved, pos=pos, pairs=pairs)
    assert check_append(st, rope) == 0


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_append_without_rotation_or_queries(cache):
    kind = "e4m3" if cache == "e4m3" else None
    assert check_append(Step([(20, 50), (1, 1)], cache=kind, held_before=False)) == 0
    rope = dict(cos_sin=make_angles(100, 64), rot=64, interleaved=False, pos=None, pairs=None)
    assert check_append(Step([(20, 50), (1, 1)], cache=kind, held_before=False), rope, with_q=False) == 0
    assert check_append(Step([(20, 50), (1, 1)], cache=kind, held_before=False), rope, in_place=True) == 0
    inter = dict(rope, interleaved=True)
    assert check_append(Step([(20, 50), (1, 1)], cache=kind, held_before=False), inter, in_place=True) == 0


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_append_skips(cache):
    """Positions beyond the table of angles, ids beyond the pool, tables that end too early."""
    kind = "e4m3" if cache == "e4m3" else None
    rope = dict(cos_sin=make_angles(40, 64), rot=64, interleaved=False, pos=None, pairs=None)
    assert check_append(Step([(20, 50), (30, 30)], cache=kind, held_before=False), rope) == B.ST_BAD_POS
    st = Step([(20, 35), (30, 30)], cache=kind, held_before=False)
    st.table[1] = st.blocks
    assert check_append(st, rope) == B.ST_BAD_BLOCK
    st = Step([(20, 35), (30, 30)], cache=kind, held_before=False)
    st.table[2] = 0xffffffff
    st.seqs[1] = (*st.seqs[1][:3], 0xffffffff)
    assert check_append(st, rope) == B.ST_BAD_BLOCK


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_append_refuses_records(cache):
    """Records that cannot be honoured: nothing of theirs is written, the others are served."""
    kind = "e4m3" if cache == "e4m3" else None
    for bad in [(5, 4, 3, 0), (38, 5, 20, 0), (0, 31, 40, 0), (0, 1, 0x80000000, 0), (0xffffffff, 1, 1, 0)]:
        st = Step([(10, 12), (30, 30)], cache=kind, held_before=False)
        st.seqs = [st.seqs[0], bad, st.seqs[1]]
        q_out, status = run_append(st, max_new=30)
        good = [st.seqs[0], st.seqs[2]]
        want_q, _ = ref.append(st.cpu, st.dtype, good, st.table, st.q, st.k, st.v, None)
        planes, scales = st.cache_back()
        assert status == B.ST_BAD_EXTENT and same(q_out, want_q), bad
        assert all(same(a, b) for a, b in zip(planes, st.cpu.planes)) and all(same(a, b) for a, b in zip(scales, st.cpu.scales))


@gpu
def test_append_e4m3_scales():
    """A block that fills token by token: scales that grow, that stay, zeros, infinities, NaN, the smallest scale."""
    T, h, d = 16, 2, 64
    st = Step([(1, 1)], T=T, h=h, group=1, d=d, cache="e4m3", held_before=False, extra_blocks=0)
    rng = np.random.default_rng(3)
    sizes = [0.0, 1e-30, 1e-3, 1.0, 448.0, 449.0, 0.875, 3e4, 1e-8, math.inf, 5.0, math.nan, 6e4, 1.0, 7.0, 2e4]
    for i, size in enumerate(sizes):
        x = rng.uniform(-1, 1, (1, h, d)).astype(np.float32)
        x[0, 1] *= 0.01
        x[0, 0, 5] = 1.0
        with np.errstate(all="ignore"):
            x = x * np.float32(size) if np.isfinite(size) else np.where(np.arange(d) == 9, np.float32(size), x)
        st.dtype = "bf16"
        st.k, st.v = ref.round16(x, "bf16"), ref.round16(-x[:, ::-1], "bf16")
        st.seqs = [(0, 1, i + 1, 0)]
        assert check_append(st) == 0, i
        if size == math.inf:
            assert ref.E4M3[st.cpu.planes[0][0, i, 0, 9]] == 448.0
    assert all((s >= 2.0 ** -64).all() for s in st.cpu.scales)
    assert np.isnan(ref.E4M3[st.cpu.planes[0][0, 11, 0, 9]])


@gpu
def test_append_is_within_its_roundings_of_64_bits():
    """Apart from the bit-exact definition: cached values against 64-bit rotation, one rounding and three 32-bit ones away."""
    rope = dict(cos_sin=make_angles(300, 128), rot=128, interleaved=False, pos=None, pairs=None)
    for dtype, kind in (("bf16", None), ("fp16", None), ("bf16", "e4m3")):
        st = Step([(200, 260)], h=2, d=128, dtype=dtype, cache=kind, held_before=False, seed=9)
        q_out, _ = run_append(st, rope)
        planes, scales = st.cache_back()
        c, s = (rope["cos_sin"][60:260, i * 64:i * 64 + 64].astype(np.float64)[:, None] for i in (0, 1))
        for x, which in ((st.q, "q"), (st.k, "k")):
            a, b = x[:, :, :64].astype(np.float64), x[:, :, 64:].astype(np.float64)
            exact = np.concatenate([a * c - b * s, b * c + a * s], 2)
            slack = 3 * ref.F32 * np.concatenate([np.abs(a * c) + np.abs(b * s)] * 2, 2) + \
                3 * ref.F32 * np.concatenate([np.abs(b * c) + np.abs(a * s)] * 2, 2)
            got = q_out
            unit, floor = ref.UNIT[dtype], 2.0 ** -25
            if which == "k":
                at = np.arange(60, 260)
                block, slot = st.table[at // 16], at % 16
                got = planes[0][block, slot].astype(np.float64)
                if kind == "e4m3":
                    got = ref.E4M3[planes[0][block, slot]] * scales[0][block][:, :, None]
                    unit, floor = 2.0 ** -4, 2.0 ** -10 * scales[0][block][:, :, None]
            assert (np.abs(got - exact) <= 1.01 * unit * np.abs(exact) + slack * 2 + floor).all()


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("rot,interleaved", [(64, False), (64, True), (62, False), (62, True), (6, False), (48, False)])
def test_append_in_place_by_every_kind_of_rotation(rot, interleaved, cache):
    """q_out is q: partners that lie in other lanes' vectors are read before any of them is written."""
    rope = dict(cos_sin=make_angles(100, rot), rot=rot, interleaved=interleaved, pos=None, pairs=None)
    for seqs in ([(20, 50), (1, 1)], [(1, 9)] * 5, [(2, 3)]):
        st = Step(seqs, h=2, group=4, cache="e4m3" if cache == "e4m3" else None, held_before=False)
        assert check_append(st, rope, in_place=True) == 0


# ---------------------------------------------------------------- attend

def run_attend(st, *, causal=True, window=0, sm_scale=None, with_lse=True, work_fill=0xff):
    t = ref.TYPES[st.dtype]
    sm_scale = 1.0 / math.sqrt(st.d) if sm_scale is None else sm_scale
    out = torch.full((max(1, st.rows), st.hq, st.d), math.nan, dtype=t, device=DEV)
    lse = torch.full((max(1, st.rows), st.hq), math.nan, device=DEV) if with_lse else None
    attn = B.make_attn(st.hq, {"bf16": B.BF16, "fp16": B.FP16}[st.dtype], sm_scale, causal=causal, window=window)
    need = B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn)
    assert need > 0
    work = torch.full((need,), work_fill, dtype=torch.uint8, device=DEV)
    B.tutti_kv_attend(st.pool, st.scales, st.batch, attn, B.make_rows(st.d_q), B.make_rows(out), lse, work, need, st.status)
    torch.cuda.synchronize()
    return out.float().cpu().numpy(), lse.cpu().numpy() if with_lse else None, int(st.status.item())


def check_attend(st, *, table_len=None, **kw):
    """Against 64 bits: every output within the error that the stated roundings allow (kv_reference.attend)."""
    out, lse, status = run_attend(st.to_gpu() if table_len is None else st, **kw)
    ref_kw = {k: v for k, v in kw.items() if k in ("causal", "window")}
    sm = kw.get("sm_scale")
    want, want_lse, err, lse_err, want_status = ref.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group,
                                                           1.0 / math.sqrt(st.d) if sm is None else sm, table_len=table_len, **ref_kw)
    assert status == want_status
    untouched = np.isnan(want_lse)
    assert np.array_equal(np.isnan(out), np.broadcast_to(untouched[:, :, None], out.shape) | np.isnan(want))
    fine = np.isfinite(want)
    assert np.array_equal(out[~fine & ~np.isnan(want)], want[~fine & ~np.isnan(want)])
    over = (np.abs(out - want) - err)[fine]
    assert over.size == 0 or over.max() <= 0, f"{over.max():.3g} beyond the bound"
    if lse is not None:
        none = want_lse == -math.inf
        assert np.array_equal(lse == -math.inf, none) and np.array_equal(np.isnan(lse), untouched)
        fine = np.isfinite(want_lse)
        assert (np.abs(lse - want_lse)[fine] <= lse_err[fine]).all()
    return out, lse


ATTEND_SHAPES = [
    [(1, 1)], [(1, 2)], [(1, 15)], [(1, 16)], [(1, 31)], [(1, 32)], [(1, 33)], [(1, 257)], [(1, 1000)], [(1, 5000)], [(2, 2)], [(5, 5)],
    [(5, 64)], [(8, 700)], [(9, 9)], [(16, 16)], [(33, 33)], [(64, 64)], [(100, 100)], [(70, 300)], [(130, 131)], [(300, 300)],
    [(0, 0), (1, 20), (0, 9)], [(1, 1 + 37 * i) for i in range(70)], [(1, 3000), (90, 200), (7, 7), (1, 1), (33, 1033)]]


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("group", [1, 4])
@pytest.mark.parametrize("seqs", ATTEND_SHAPES, ids=lambda s: "-".join(f"{a}of{b}" for a, b in s[:5]))
def test_attend_lengths(seqs, group, cache):
    check_attend(Step(seqs, group=group, cache="e4m3" if cache == "e4m3" else None, seed=len(seqs)))


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T,h,group,d,hnd,dtype,gap", [
    (16, 8, 4, 128, False, "bf16", 0), (16, 8, 4, 128, True, "fp16", 48), (32, 1, 8, 128, True, "bf16", 16), (64, 5, 1, 80, False, "fp16", 0),
    (128, 2, 16, 96, True, "bf16", 0), (48, 3, 5, 112, False, "bf16", 0), (16, 2, 33, 64, False, "bf16", 0), (1, 2, 3, 16, False, "fp16", 0),
    (5, 4, 1, 96, True, "bf16", 16), (8, 1, 7, 32, False, "fp16", 32), (17, 2, 2, 128, False, "bf16", 48), (20, 1, 4, 48, True, "fp16", 0)])
def test_attend_layouts(cache, T, h, group, d, hnd, dtype, gap):
    for seqs in ([(1, 700), (1, 1), (1, 45)], [(4, 300), (1, 7)], [(1, 130), (100, 210), (9, 9)]):
        check_attend(Step(seqs, T=T, h=h, group=group, d=d, dtype=dtype, hnd=hnd, gap=gap, pad_rows=1,
                          cache="e4m3" if cache == "e4m3" else None, seed=T + d))


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("window", [1, 2, 31, 32, 33, 100, 4096])
def test_attend_window(window, cache):
    """Blocks behind the window may be anything: their ids are taken out of the table."""
    for seqs in ([(1, 1000), (1, 40)], [(6, 333)], [(150, 400), (1, 200), (40, 40)]):
        st = Step(seqs, cache="e4m3" if cache == "e4m3" else None, seed=window)
        for _, n_new, n_held, off in st.seqs:
            gone = max(0, n_held - n_new + 1 - window) // st.T
            st.table[off:off + gone] = 0xffffffff
        check_attend(st, window=window)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 24])
def test_attend_not_causal_and_scales(T, cache):
    kind = "e4m3" if cache == "e4m3" else None
    check_attend(Step([(20, 45), (1, 300), (70, 70)], T=T, cache=kind), causal=False)
    check_attend(Step([(20, 45), (1, 300), (70, 70)], T=T, cache=kind), sm_scale=0.0, with_lse=False)
    check_attend(Step([(20, 45), (1, 300), (70, 70)], T=T, cache=kind), sm_scale=-1.5)
    check_attend(Step([(20, 45), (1, 600), (70, 70)], T=T, cache=kind, spread=6.0))


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("T", [16, 12])
def test_attend_blocks_that_are_not_there(T, cache):
    """Ids beyond the pool and a table that ends early: those keys are not seen; a row may see none at all."""
    for seqs in ([(1, 500), (1, 10)], [(3, 90), (40, 200)]):
        st = Step(seqs, T=T, cache="e4m3" if cache == "e4m3" else None)
        st.table[2], st.table[5] = st.blocks, 0xffffffff
        check_attend(st)
        st = Step(seqs, T=T, cache="e4m3" if cache == "e4m3" else None)
        st.to_gpu()
        st.set_batch(table_len=len(st.table) - 2)
        check_attend(st, table_len=len(st.table) - 2)
    st = Step([(1, 40), (9, 9)], T=T, cache="e4m3" if cache == "e4m3" else None)
    st.table[:] = 0xffffffff
    out, lse = check_attend(st)
    assert (out == 0).all() and (lse == -math.inf).all()


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
@pytest.mark.parametrize("n_new", [5, 60])
@pytest.mark.parametrize("T", [16, 10])
def test_attend_values_that_are_not_finite(T, n_new, cache):
    """A NaN or an infinity among the values reaches the queries that see it, and no other."""
    st = Step([(n_new, n_new + 30)], T=T, cache="e4m3" if cache == "e4m3" else None, d=128)
    at = 30 + 3
    block = st.table[at // T]
    st.cpu.planes[1][block, at % T, 1, 7] = 0x7f if cache == "e4m3" else math.inf
    out, _, _ = run_attend(st.to_gpu())
    for i in range(n_new):
        for head in range(st.hq):
            x = out[i, head]
            hit = i >= 3 and head // st.group == 1
            assert np.isfinite(np.delete(x, 7)).all() and np.isfinite(x[7]) != hit, (i, head)
    # keys: a NaN score makes the whole row NaN, where it is seen
    st = Step([(n_new, n_new + 30)], T=T, cache="e4m3" if cache == "e4m3" else None, d=128)
    st.cpu.planes[0][block, at % T, 0, 3] = 0x7f if cache == "e4m3" else math.nan
    out, _, _ = run_attend(st.to_gpu())
    for i in range(n_new):
        for head in range(st.hq):
            assert np.isnan(out[i, head]).all() == (i >= 3 and head // st.group == 0) and \
                np.isnan(out[i, head]).any() == (i >= 3 and head // st.group == 0), (i, head)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_attend_large_scores(cache):
    """Scores of some thousands, and values' scales far apart: maxima do their work."""
    st = Step([(1, 700), (6, 90)], cache="e4m3" if cache == "e4m3" else None)
    st.q = ref.round16(st.q * 300, st.dtype)
    check_attend(st)
    if cache == "e4m3":
        st = Step([(1, 700), (40, 90)], cache="e4m3")
        for scales in st.cpu.scales:
            scales *= np.exp2(np.random.default_rng(1).integers(-12, 12, scales.shape)).astype(np.float32)
        check_attend(st, sm_scale=0.01)


@gpu
@pytest.mark.parametrize("cache", ["16", "e4m3"])
def test_attend_refuses_records(cache):
    kind = "e4m3" if cache == "e4m3" else None
    for bad in [(5, 4, 3, 0), (38, 5, 20, 0), (0, 31, 40, 0), (0, 1, 0x80000000, 0), (0xffffffff, 1, 1, 0)]:
        st = Step([(10, 12), (30, 30)], cache=kind)
        st.seqs = [st.seqs[0], bad, st.seqs[1]]
        st.to_gpu()
        st.set_batch(max_new=30)
        out, lse, status = run_attend(st)
        assert status == B.ST_BAD_EXTENT, bad
        st.seqs = [st.seqs[0], st.seqs[2]]
        want, _, err, _, _ = ref.attend(st.cpu, st.dtype, st.seqs, st.table, st.q, st.group, 1.0 / math.sqrt(st.d))
        assert (np.abs(out - want) <= err).all()


@gpu
def test_attend_twice_the_same():
    """No result depends on which workgroup ends first; the work memory's contents do not matter."""
    st = Step([(1, 3000), (1, 500), (2, 40)], h=8, d=128, cache="e4m3").to_gpu()
    first = run_attend(st, work_fill=0xff)
    for fill in (0x00, 0x7f, 0x3c):
        again = run_attend(st, work_fill=fill)
        assert same(first[0], again[0]) and same(first[1], again[1])


@gpu
def test_on_another_stream_and_in_a_graph():
    """Both calls on a stream of the caller's and replayed from a captured graph, the work memory used by others between."""
    st = Step([(1, 900), (1, 40), (3, 20)], h=4, group=4, d=128, cache="e4m3", held_before=False).to_gpu()
    rope = B.make_rope(torch.from_numpy(make_angles(1000, 128)).to(DEV), 128)
    t = ref.TYPES[st.dtype]
    q_out = torch.empty((st.rows, st.hq, st.d), dtype=t, device=DEV)
    out, lse = torch.empty_like(q_out), torch.empty((st.rows, st.hq), device=DEV)
    attn = B.make_attn(st.hq, B.BF16, 0.1)
    work = torch.empty(B.tutti_kv_attend_work_bytes(st.pool, st.batch, attn), dtype=torch.uint8, device=DEV)

    def step():
        B.tutti_kv_append(st.pool, st.scales, st.batch, rope, B.make_rows(st.d_q), B.make_rows(q_out), B.make_rows(st.d_k),
                          B.make_rows(st.d_v), st.hq, B.BF16)
        B.tutti_kv_attend(st.pool, st.scales, st.batch, attn, B.make_rows(q_out), B.make_rows(out), lse, work, work.numel())

    step()
    torch.cuda.synchronize()
    want, want_lse = out.clone(), lse.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out.fill_(0)
    lse.fill_(0)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    assert torch.equal(out, want) and torch.equal(lse, want_lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        out.fill_(i)
        work.fill_(17 * i)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(lse, want_lse)
        step()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


@gpu
def test_offsets_beyond_32_bits():
    """A pool of more than 4 GiB a plane, blocks at both ends of it, and a table offset beyond the first sequences."""
    T, h, d = 16, 8, 128
    stride = 1 << 20
    blocks = 4200                                              # 4.1 GiB a plane
    rng = np.random.default_rng(2)
    planes = [torch.zeros(blocks * stride, dtype=torch.uint8, device=DEV) for _ in range(2)]
    pool = B.make_pool(*planes, num_blocks=blocks, block_tokens=T, num_kv_heads=h, head_dim=d, elt_bytes=2, block_stride=stride)
    ids = np.array([4199, 0, 4100, 4097, 1, 4198], np.uint32)
    n = 6 * T - 3
    k, v = (ref.round16(rng.standard_normal((n, h, d)), "bf16") for _ in range(2))
    q = ref.round16(rng.standard_normal((n, h, d)), "bf16")
    dev = [torch.from_numpy(x).to(torch.bfloat16).to(DEV) for x in (q, k, v)]
    seqs = torch.tensor([[0, n, n, 2]], dtype=torch.int32, device=DEV)
    table = torch.from_numpy(np.concatenate([[9, 9], ids]).astype(np.int32)).to(DEV)
    batch = B.make_batch(seqs, 1, n, table, table.numel(), n)
    B.tutti_kv_append(pool, None, batch, None, None, None, B.make_rows(dev[1]), B.make_rows(dev[2]), 0, B.BF16)
    attn = B.make_attn(h, B.BF16, 0.05)
    out, lse = torch.empty_like(dev[0]), torch.empty((n, h), device=DEV)
    work = torch.empty(B.tutti_kv_attend_work_bytes(pool, batch, attn), dtype=torch.uint8, device=DEV)
    B.tutti_kv_attend(pool, None, batch, attn, B.make_rows(dev[0]), B.make_rows(out), lse, work, work.numel())
    torch.cuda.synchronize()
    for plane, x in zip(planes, (dev[1], dev[2])):
        got = plane.view(blocks, stride)[torch.from_numpy(ids.astype(np.int64)).to(DEV), :T * h * d * 2].contiguous()
        assert torch.equal(got.view(torch.bfloat16).view(6 * T, h, d)[:n], x)
    cache = ref.Cache(6, T, h, d, "bf16")
    for plane, x in zip(cache.planes, (k, v)):
        plane.reshape(6 * T, h, d)[:n] = x
    want, want_lse, err, lse_err, _ = ref.attend(cache, "bf16", [(0, n, n, 0)], np.arange(6), q, 1, 0.05)
    assert (np.abs(out.float().cpu().numpy() - want) <= err).all() and (np.abs(lse.cpu().numpy() - want_lse) <= lse_err).all()


# ---------------------------------------------------------------- the reference itself, and refusals (CPU)

def test_reference_e4m3():
    values = ref.E4M3[np.isfinite(ref.E4M3)]
    assert values.max() == 448.0 and (ref.E4M3[ref.to_e4m3(values)] == values).all()
    x = np.random.default_rng(0).uniform(-460, 460, 4000) * 2.0 ** np.random.default_rng(1).integers(-18, 1, 4000)
    theirs = torch.from_numpy(np.clip(x, -448, 448)).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(ref.to_e4m3(x), theirs)
    assert ref.scale_for([448.0]) == 1.0 and ref.scale_for([448.1]) == 2.0 and ref.scale_for([0.0]) == 2.0 ** -64


GOOD = dict(num_blocks=8, block_tokens=16, num_kv_heads=2, head_dim=64, elt_bytes=2)


def _code(fn, *a):
    try:
        return fn(*a, stream=0)
    except B.TuttiError as e:
        return e.code


def _append_args(**kw):
    pool = B.make_pool(kw.get("k_base", FAKE), FAKE, **dict(GOOD, **kw.get("pool", {})))
    rows = {n: B.make_rows(FAKE, 1024, 128) for n in ("q", "q_out", "k", "v")}
    rows.update(kw.get("rows", {}))
    rope = B.make_rope(FAKE, 64, n_pos=10)
    for name, x in kw.get("rope", {}).items():
        setattr(rope, name, x)
    batch = B.make_batch(FAKE, 0, 1, FAKE, 4, 1)                     # no sequence: accepted, nothing enqueued
    for name, x in kw.get("batch", {}).items():
        setattr(batch, name, x)
    return (pool, kw.get("scales"), batch, rope, rows["q"], rows["q_out"], rows["k"], rows["v"], kw.get("heads", 4),
            kw.get("dtype", B.BF16), kw.get("status", 0))


SCALES = B.make_scales(FAKE, FAKE, 4)
BAD_POOLS = [dict(num_blocks=0), dict(head_dim=0), dict(head_dim=24), dict(head_dim=144), dict(block_tokens=0), dict(num_kv_heads=0),
             dict(elt_bytes=4), dict(elt_bytes=1), dict(block_stride=4000), dict(block_stride=4104), dict(pool_layout=2),
             dict(block_tokens=1 << 30, num_kv_heads=64)]


def test_append_refuses():
    assert _code(B.tutti_kv_append, *_append_args()) == B.OK
    assert _code(B.tutti_kv_append, *_append_args(pool=dict(elt_bytes=1), scales=SCALES)) == B.OK
    axes = (B.C.c_uint32 * 4)(10, 20, 1, 0)
    bad = [dict(pool=p) for p in BAD_POOLS] + [
        dict(k_base=0), dict(k_base=FAKE + 8), dict(scales=SCALES), dict(dtype=0), dict(dtype=3), dict(status=FAKE + 2),
        dict(pool=dict(elt_bytes=1), scales=B.make_scales(0, FAKE, 4)), dict(pool=dict(elt_bytes=1), scales=B.make_scales(FAKE + 2, FAKE, 4)),
        dict(pool=dict(elt_bytes=1), scales=B.make_scales(FAKE, FAKE, 1)), dict(heads=0),
        dict(batch=dict(n_seq=1, d_seqs=0)), dict(batch=dict(n_seq=1, d_seqs=FAKE + 8)), dict(batch=dict(n_seq=1, d_block_table=0)),
        dict(rope=dict(rot_dim=0)), dict(rope=dict(rot_dim=3)), dict(rope=dict(rot_dim=66)), dict(rope=dict(d_cos_sin=0)),
        dict(rope=dict(d_cos_sin=FAKE + 4)), dict(rope=dict(n_pos=0)), dict(rope=dict(interleaved=2)), dict(rope=dict(d_pos=FAKE + 2)),
        dict(rope=dict(d_pos=FAKE, axis_pairs=axes))]
    for name in ("k", "v", "q_out"):
        for rows in (B.make_rows(0, 1024, 128), B.make_rows(FAKE + 8, 1024, 128), B.make_rows(FAKE, 1032, 128), B.make_rows(FAKE, 1024, 136),
                     None):
            bad.append(dict(rows={name: rows}))
    for kw in bad:
        assert _code(B.tutti_kv_append, *_append_args(**kw)) == B.EINVAL, kw
    assert _code(B.tutti_kv_append, *_append_args(batch=dict(n_seq=B.MAX_REQ + 1))) == B.ERANGE
    assert _code(B.tutti_kv_append, *_append_args(batch=dict(n_rows=1 << 31))) == B.ERANGE
    assert _code(B.tutti_kv_append, *_append_args(heads=1 << 16)) == B.ERANGE
    assert _code(B.tutti_kv_append, *_append_args(rows=dict(q=None, q_out=None), heads=0)) == B.OK
    for none in range(3):
        args = list(_append_args())
        args[[0, 2, 6][none]] = None
        assert _code(B.tutti_kv_append, *args) == B.EINVAL


def test_attend_refuses():
    def args(**kw):
        pool, scales, batch, _, q, out, *_ = _append_args(**{k: v for k, v in kw.items() if k != "attn"})
        attn = B.make_attn(4, kw.get("dtype", B.BF16), 0.1)
        for name, x in kw.get("attn", {}).items():
            setattr(attn, name, x)
        return pool, scales, batch, attn, q, out, kw.get("lse", 0), kw.get("work", FAKE), kw.get("bytes", 1 << 40), kw.get("status", 0)

    assert _code(B.tutti_kv_attend, *args()) == B.OK
    bad = [dict(pool=p) for p in BAD_POOLS] + [
        dict(scales=SCALES), dict(dtype=0), dict(attn=dict(n_q_heads=0)), dict(attn=dict(n_q_heads=5)), dict(attn=dict(sm_scale=math.inf)),
        dict(attn=dict(sm_scale=math.nan)), dict(attn=dict(causal=2)), dict(attn=dict(causal=0, window=5)), dict(lse=FAKE + 2),
        dict(status=FAKE + 1), dict(batch=dict(n_seq=1, d_seqs=FAKE + 4)), dict(batch=dict(n_seq=1), work=0),
        dict(batch=dict(n_seq=1), work=FAKE + 8), dict(rows=dict(q=B.make_rows(FAKE, 1000, 128))), dict(rows=dict(q_out=None))]
    for kw in bad:
        assert _code(B.tutti_kv_attend, *args(**kw)) == B.EINVAL, kw
    pool, _, batch, attn, *_ = args(batch=dict(n_seq=1))
    need = B.tutti_kv_attend_work_bytes(pool, batch, attn)
    assert need > 0 and _code(B.tutti_kv_attend, *args(batch=dict(n_seq=1), bytes=need - 1)) == B.ERANGE
    assert _code(B.tutti_kv_attend, *args(batch=dict(n_seq=B.MAX_REQ + 1))) == B.ERANGE
    assert B.tutti_kv_attend_work_bytes(pool, batch, B.make_attn(5, B.BF16, 0.1)) == 0
    assert B.tutti_kv_attend_work_bytes(None, batch, attn) == 0
    for x in (torch.zeros(2, 3), torch.zeros(2, 3, 4).transpose(1, 2)):
        with pytest.raises(ValueError):
            B.make_rows(x)
    with pytest.raises(ValueError):
        B.make_scales(torch.zeros(4, 4), torch.zeros(4, 8))


def test_work_bytes_refuses_what_the_call_refuses():
    """Shapes, types and counts; not what only the call is handed (addresses, scales)."""
    def size(pool=(), batch=(), attn=()):
        p, b = B.make_pool(0, 0, **dict(GOOD, **dict(pool))), B.make_batch(0, 1, 1, 0, 4, 1)
        a = B.make_attn(4, B.BF16, 0.1)
        for record, fields in ((b, batch), (a, attn)):
            for name, x in dict(fields).items():
                setattr(record, name, x)
        return B.tutti_kv_attend_work_bytes(p, b, a)

    assert size() > 0 and size(pool=dict(elt_bytes=1)) > 0
    for bad in BAD_POOLS:
        if bad != dict(elt_bytes=1):        # (without scales: the call's matter)
            assert size(pool=bad) == 0, bad
    for bad in (dict(n_seq=B.MAX_REQ + 1), dict(n_rows=1 << 31), dict(n_rows=(1 << 31) - 1)):
        assert size(batch=bad) == 0, bad
    for bad in (dict(dtype=0), dict(dtype=3), dict(n_q_heads=0), dict(n_q_heads=5), dict(sm_scale=math.inf), dict(causal=2),
                dict(causal=0, window=5)):
        assert size(attn=bad) == 0, bad
    assert B.tutti_kv_attend_work_bytes(B.make_pool(0, 0, **GOOD), None, B.make_attn(4, B.BF16, 0.1)) == 0
    assert B.tutti_kv_attend_work_bytes(B.make_pool(0, 0, **GOOD), B.make_batch(0, 1, 1, 0, 4, 1), None) == 0


def test_more_threads_than_a_launch_has():
    """2^32 threads and more: refused as such, before anything is launched."""
    big = dict(n_seq=1, max_new=2)
    for rows, pool in (((1 << 29) - 1, {}), (1 << 30, {}), ((1 << 31) - 1, {}), (1 << 30, dict(elt_bytes=1))):
        args = _append_args(batch=dict(big, n_rows=rows), pool=pool, scales=SCALES if pool else None)
        assert _code(B.tutti_kv_append, *args) == B.ERANGE, rows
    for max_new, heads, rows in ((1, 2, 1 << 29), (20, 2, 1 << 28), (64, 2, (1 << 30) - 1)):
        pool, _, batch, _, q, out, *_ = _append_args(batch=dict(n_seq=1, max_new=max_new, n_rows=rows))
        attn = B.make_attn(heads, B.BF16, 0.1)
        threads = (rows * heads // 2 // (16 if max_new == 1 else 32 if max_new == 20 else 128) + 1) * (1 if max_new < 64 else 2) * 256
        refused = threads >= 1 << 32
        assert (B.tutti_kv_attend_work_bytes(pool, batch, attn) == 0) == refused, max_new
        if refused:
            assert _code(B.tutti_kv_attend, pool, None, batch, attn, q, out, 0, FAKE, 1 << 60) == B.ERANGE, max_new


# ---------------------------------------------------------------- together, with the calls that move blocks

@gpu
def test_example_decodes_over_a_restored_prefix():
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "decode_after_restore.py")
    spec = importlib.util.spec_from_file_location("decode_after_restore", path)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    a, b = example.run(prompts=(200, 33, 16), chunk=96, steps=18)
    assert a.shape == (18, 3, example.HQ, example.D) and torch.isfinite(a.float()).all() and torch.equal(a, b)
