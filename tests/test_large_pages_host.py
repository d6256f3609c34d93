"""Pages and blocks larger than the kernels count are refused, without a GPU (fake addresses are never dereferenced)."""
import ctypes as C

import pytest

from oracle import kv_oracle as O
from tests.test_cache4_host import CLOSED, E2M1, _at, _desc, kv, no_gpu      # noqa: F401 (fixtures)


@pytest.mark.parametrize("elem", [E2M1, 1, 2])
def test_pages_of_two_gigabytes_are_not_moved(kv, no_gpu, elem):
    lib = kv.load()
    ids, offs = (C.c_int32 * 2)(3, 5), (C.c_int32 * 2)(0, 2)
    wires = (C.c_void_p * 1)(_at(1))
    logical, table, merged = (C.c_int32 * 2)(0, 1), (C.c_int32 * 1)(), (C.c_int32 * 2)()

    def calls(block_size):
        desc = _desc(elem, block_size=block_size, n_kv_heads=1)
        assert desc.block_stride == kv.kv_cache_page_bytes(block_size, 1, 128, 0.5 if elem == E2M1 else elem)
        return {lib.kv_pack_blocks(C.byref(desc), ids, 2, _at(1), 1 << 50, 0, 0),
                lib.kv_unpack_assemble(C.byref(desc), _at(1), 1 << 50, 0, logical, ids, 2, table, 0, 2 * block_size if block_size < 1 << 30 else 0,
                                       1, 1, merged, 0),
                lib.kv_pack_blocks_batched(C.byref(desc), 1, offs, ids, wires, 0, 0),
                lib.kv_unpack_blocks_batched(C.byref(desc), 1, offs, ids, wires, 0, 0)}
    row = {E2M1: 73, 1: 129, 2: 256}[elem]
    fits = 0x7fff0000 // row // 16 * 16
    assert calls(fits) == {CLOSED}
    assert calls(fits + 16) == calls((1 << 31) // row + 16) == calls((1 << 32) // row // 16 * 16 + 16) == {O.ERR_SHAPE}


@pytest.mark.parametrize("elem", [E2M1, 1, 2])
def test_bounds_count_keys_in_32_bits(kv, no_gpu, elem):
    lib = kv.load()

    def call(block_size):
        return lib.kv_op_block_bounds(C.byref(_desc(elem, block_size=block_size, n_kv_heads=1)), 0, _at(1), _at(2), 3, _at(3), _at(4), 0)
    assert call(1 << 30) == CLOSED
    assert call((1 << 30) + 1) == call((1 << 31) - 16) == call((1 << 31) - 1) == O.ERR_SHAPE
