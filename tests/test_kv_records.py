"""CPU tests of the helpers that make the records of the calls on a paged cache from tensors: what the kernels would misread is refused."""
import pytest
import torch

from paper_2605_03375_amd import binding as B


def test_rope_of_tensors():
    cos_sin, pos = torch.zeros(40, 64), torch.zeros(3, 9, dtype=torch.int32)
    r = B.make_rope(cos_sin, 64)
    assert (r.d_cos_sin, r.n_pos, r.d_pos, tuple(r.axis_pairs)) == (cos_sin.data_ptr(), 40, None, (32, 0, 0, 0))
    r = B.make_rope(cos_sin, 64, d_pos=pos, pairs=(8, 12, 12))
    assert (r.d_pos, r.pos_stride, tuple(r.axis_pairs)) == (pos.data_ptr(), 9, (8, 12, 12, 0))
    r = B.make_rope(cos_sin, 64, d_pos=torch.zeros(3, 20, dtype=torch.int32)[:, :9], pairs=(8, 12, 12))
    assert r.pos_stride == 20
    r = B.make_rope(cos_sin, 64, n_pos=30, d_pos=pos[0], pairs=(32,))       # one axis, without a dimension of its own
    assert (r.n_pos, r.pos_stride) == (30, 9)
    assert B.make_rope(torch.zeros(40 * 64), 64, n_pos=40).n_pos == 40
    r = B.make_rope(0x10000, 64, n_pos=7, d_pos=0x20000, pos_stride=5, pairs=(16, 16))
    assert (r.d_cos_sin, r.n_pos, r.d_pos, r.pos_stride) == (0x10000, 7, 0x20000, 5)


@pytest.mark.parametrize("bad", [
    torch.zeros(40, 64, dtype=torch.bfloat16), torch.zeros(40, 64, dtype=torch.float64), torch.zeros(40, 64, dtype=torch.int32),
    torch.zeros(40, 32), torch.zeros(40, 128)[:, :64], torch.zeros(64, 40).T, torch.zeros(40 * 64), torch.zeros(40, 128)])
def test_angles_that_are_no_table(bad):
    """Rows of another type or length, or apart: the kernel would read beyond them."""
    with pytest.raises(ValueError):
        B.make_rope(bad, 64)


def test_counts_that_are_wrong_or_missing():
    for bad in (dict(n_pos=41), dict(d_cos_sin=0x10000), dict(d_pos=0x10000)):
        with pytest.raises(ValueError):
            B.make_rope(**dict(dict(d_cos_sin=torch.zeros(40, 64), rot_dim=64), **bad))


@pytest.mark.parametrize("bad", [
    torch.zeros(3, 9, dtype=torch.int64), torch.zeros(3, 9, dtype=torch.int16), torch.zeros(3, 9), torch.zeros(9, 3, dtype=torch.int32).T,
    torch.zeros(2, 9, dtype=torch.int32), torch.zeros(9, dtype=torch.int32), torch.zeros(3, 9, 1, dtype=torch.int32)])
def test_positions_that_are_not_32_bits_by_axis(bad):
    with pytest.raises(ValueError):
        B.make_rope(torch.zeros(40, 64), 64, d_pos=bad, pairs=(8, 12, 12))


def test_rows_of_tensors():
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16)
    r = B.make_rows(x[:, 1:3])
    assert (r.base, r.row_stride, r.head_stride) == (x.data_ptr() + 128, 512, 128)
    for dtype in (torch.float32, torch.float64, torch.int8, torch.int16):
        with pytest.raises(ValueError):
            B.make_rows(x.to(dtype))


def test_scales_of_tensors():
    k = torch.zeros(6, 8)
    s = B.make_scales(k, k.clone())
    assert s.stride == 8
    for bad in (torch.zeros(6, 8, dtype=torch.int32), torch.zeros(6, 8, dtype=torch.float16), torch.zeros(6), torch.zeros(8, 6).T):
        with pytest.raises(ValueError):
            B.make_scales(bad, bad)
    with pytest.raises(ValueError):
        B.make_scales(k, k.to(torch.int32))
