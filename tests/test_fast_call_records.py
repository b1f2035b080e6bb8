"""CPU tests of what the extension module takes for the records of the calls on a paged cache: the record or None, nothing else."""
import ctypes as C

import pytest
import torch

from paper_2605_03375_amd import binding as B
from paper_2605_03375_amd import build

RECORDS = {"scales": B.tutti_scales, "batch": B.tutti_batch, "rope": B.tutti_rope, "attn": B.tutti_attn, "q": B.tutti_rows,
           "q_out": B.tutti_rows, "out": B.tutti_rows, "k": B.tutti_rows, "v": B.tutti_rows}


@pytest.fixture
def call_of():
    """For an entry point: a callable bound to a recorder, the words that arrived, the calls left to the wrapper, good arguments."""
    build.build_fast_call(force=False)
    from paper_2605_03375_amd import _fast_call as module
    lib = B.product_lib()
    module.setup(B._RECORDS, torch.Tensor, lambda: 0, lambda device: 5, B._check)
    module.enable(True)
    keep = []

    def make(name):
        types = [t if t in (C.c_uint32, C.c_uint64) else C.c_void_p for t in getattr(lib, name).argtypes]
        got, left, wrapper = [], [], getattr(B, name)
        fn = C.CFUNCTYPE(C.c_int, *types)(lambda *a: got.append(a) or 0)
        names = wrapper.__code__.co_varnames[:wrapper.__code__.co_argcount]
        call = module.wrap(name, lambda *a: left.append(a), names, wrapper.__defaults__)
        module.bind(call, C.cast(fn, C.c_void_p).value)
        keep.append(fn)
        pool = B.make_pool(None, None, num_blocks=4, block_tokens=16, num_kv_heads=2, head_dim=64, elt_bytes=2)
        args = [pool if n == "pool" else RECORDS[n]() if n in RECORDS else 9 for n in names]
        return call, got, left, names, args
    yield make
    module.enable(False)
    B._bind_fast_calls()


@pytest.mark.parametrize("name", ["tutti_kv_append", "tutti_kv_attend"])
def test_records_and_none(call_of, name):
    call, got, left, names, args = call_of(name)
    assert call(*args) == 0 and not left
    words = got.pop()
    for n, x, word in zip(names, args, words):
        assert word == (9 if x == 9 else C.addressof(x)), n
    for i, n in enumerate(names):
        if n in RECORDS:
            assert call(*args[:i], None, *args[i + 1:]) == 0 and not left
            assert got.pop() == (*words[:i], None, *words[i + 1:]), n


@pytest.mark.parametrize("name", ["tutti_kv_append", "tutti_kv_attend"])
def test_what_is_no_record_is_left_to_the_wrapper(call_of, name):
    """A tensor's address, an integer or another record would be read as the record, in host memory."""
    call, got, left, names, args = call_of(name)
    for i, n in enumerate(names):
        if n not in RECORDS:
            continue
        for x in (torch.zeros(4, 2, 64), 4096, args[0], C.byref(args[i]), (RECORDS[n] * 1)()):
            given = [*args[:i], x, *args[i + 1:]]
            call(*given)
            a = left.pop()
            assert not got and len(a) == len(given) and all(p is q for p, q in zip(a, given)), (n, x)


def test_a_tensor_in_place_of_rows_is_an_error():
    """By ctypes and, where there is a GPU, by the module alike."""
    pool = B.make_pool(0x10000, 0x10000, num_blocks=4, block_tokens=16, num_kv_heads=2, head_dim=64, elt_bytes=2)
    batch, rows, x = B.make_batch(0x10000, 0, 1, 0x10000, 4, 1), B.make_rows(0x10000, 1024, 128), torch.zeros(4, 2, 64)
    for bad in (x, 4096, pool):
        with pytest.raises((TypeError, C.ArgumentError)):
            B.tutti_kv_append(pool, None, batch, None, rows, rows, bad, rows, 2, B.BF16, stream=0)
        with pytest.raises((TypeError, C.ArgumentError)):
            B.tutti_kv_attend(pool, None, batch, B.make_attn(2, B.BF16, 0.1), rows, bad, None, 0x10000, 1 << 30, stream=0)
