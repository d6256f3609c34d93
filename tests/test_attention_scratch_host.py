"""Scratch of the batched attention by page format, without a GPU (fake addresses are never dereferenced; 148 SMs without one)."""
import ctypes as C

import pytest

from oracle import kv_oracle as O
from tests.test_cache4_host import CLOSED, E2M1, _at, _desc, kv, no_gpu      # noqa: F401 (fixtures)


def _bytes(n_req, hq, dim, ranges):
    up = lambda x: -(-x // 256) * 256
    return up(8 * (n_req + 1)) + up(hq * ranges * 2 * 8) + up(hq * ranges * 2 * dim * 4)


@pytest.mark.parametrize("selected", [False, True])
@pytest.mark.parametrize("elem,dtype,ctas", [(2, 0, 2), (2, 1, 2), (1, 0, 2), (1, 1, 2), (E2M1, 1, 2), (E2M1, 0, 3)])
@pytest.mark.parametrize("r", [8, 32])
def test_a_call_asks_for_the_scratch_of_its_own_ranges(kv, no_gpu, r, elem, dtype, ctas, selected):
    """Two CTAs an SM, three over e2m1 pages with bf16 queries, cut each KV head's contexts into as many ranges; a buffer for those is
    enough, and what the size function says is enough for every format."""
    lib, hq, hkv, dim, ctx = kv.load(), 64, 8, 128, 4096
    q, tab, lens, scr, out = (_at(i) for i in range(1, 6))
    desc = _desc(elem, n_kv_heads=hkv)

    def call(need):
        if selected:
            return lib.kv_op_paged_attention_selected(q, hq * dim, dtype, r, hq, C.byref(desc), 0, tab, hkv * ctx // 16, ctx // 16, lens, ctx,
                                                      0.1, scr, need, out, hq * dim, None, 0)
        return lib.kv_op_paged_attention_batched(q, hq * dim, dtype, r, hq, C.byref(desc), 0, tab, ctx // 16, lens, ctx, 0.1, scr, need, out,
                                                 hq * dim, None, 0)
    need = _bytes(r, hq, dim, ctas * 148 // hkv)
    assert call(need) == CLOSED and call(need - 1) == O.ERR_WORKSPACE
    assert lib.kv_paged_attention_batched_scratch_bytes(r, hq, hkv, dim, ctx) == _bytes(r, hq, dim, 3 * 148 // hkv)
