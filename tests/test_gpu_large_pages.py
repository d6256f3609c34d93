"""e2m1 pages of so many slots that a slot's place in its page passes 32 bits."""
import numpy as np
import pytest

from oracle import pages4_oracle as P
from tests.test_gpu_serving_ops import _np, _shape

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def kv():
    import paper_2608_16477_b200 as kv
    kv.load()
    return kv


@pytest.fixture(scope="module")
def torch():
    import torch
    return torch


def test_rows_at_the_end_of_a_huge_page(kv, torch):
    """Scales of 16 dims lie 8 bytes a slot apart: from slot 2^28 on their places pass 31 bits."""
    block, d = (1 << 28) + 64, 128
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 50 << 30:
        pytest.skip("memory for one page of K and one of V")
    cache = kv.PagedCache(_shape(1, d, block), 1, elem_bytes=0.5)
    places = [0, 1, (1 << 28) - 1, 1 << 28, (1 << 28) + 1, block - 1]
    slots = torch.tensor(places, device="cuda")
    rng = np.random.default_rng(1)
    x = rng.standard_normal((2, len(places), 1, d)).astype(np.float32) * 2.0 ** rng.integers(-5, 5, (2, len(places), 1, 1)).astype(np.float32)
    k, v = torch.from_numpy(x).cuda()
    other = torch.zeros(2, len(places), 1, d, device="cuda")
    for write in ("write", "append"):
        if write == "write":
            kv.kv_op_cache_write(cache, 0, k, v, slots)
        else:
            kv.kv_op_cache_write(cache, 0, other[0], other[1], slots)
            kv.kv_op_cache_append(kv.Rope(d), cache, 0, k, v, torch.zeros(len(places), dtype=torch.int32, device="cuda"), slots)      # not turned
        ks, vs = torch.empty_like(k), torch.empty_like(v)
        kv.kv_op_cache_read(cache, 0, slots, ks, vs)
        for got, rows in ((ks, x[0]), (vs, x[1])):
            for i in range(len(places)):
                assert np.array_equal(_np(got)[i, 0], P.stored(rows[i, 0])), (write, places[i])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_at_the_end_of_a_huge_page(kv, torch, dtype):
    """Codes lie 64 bytes a slot apart: from slot 2^25 on their places pass 31 bits.  All keys are zero but a few at the end, whose weight
    is that of all others together; the bound is that of the batched attention's tests, with the sums of equal weights counted exactly."""
    n, d, group = (1 << 25) + 100, 128, 4
    block = n + 12
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 8 << 30:
        pytest.skip("memory for one page of K and one of V")
    cache = kv.PagedCache(_shape(1, d, block), 1, elem_bytes=0.5, fill=0)
    places = np.array([5, (1 << 25) - 1, 1 << 25, (1 << 25) + 17, n - 1])
    rng = np.random.default_rng(2)
    rows = torch.from_numpy(rng.uniform(0.5, 2, (2, len(places), 1, d)).astype(np.float32)).cuda()
    slots = torch.from_numpy(places).cuda()
    kv.kv_op_cache_write(cache, 0, rows[0], rows[1], slots)
    kv.kv_op_cache_read(cache, 0, slots, rows[0], rows[1])
    q = torch.full((1, group, d), 0.875, device="cuda", dtype=getattr(torch, dtype))
    scale = 20.0 / float((rows[0].sum(-1) * 0.875).max())                     # e^20: the few are much of the sum
    out, lse = torch.empty_like(q), torch.empty(1, group, device="cuda")
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(1, group, cache, n), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, torch.zeros(1, 1, dtype=torch.int32, device="cuda"),
                                     torch.tensor([n], dtype=torch.int32, device="cuda"), n, out, scratch, lse=lse, softmax_scale=scale)
    k, v = _np(rows[0])[:, 0], _np(rows[1])[:, 0]
    s = k @ _np(q)[0, 0] * scale
    p = np.exp(s)
    total = p.sum() + (n - len(places))                                       # zero keys weigh 1, and their values are zero
    want, half = p @ v / total, torch.finfo(getattr(torch, dtype)).eps / 2
    share = 20 * 2.0 ** -13 + 2.0 ** -14 + (n / 148 / 16 + 64) * 2.0 ** -22   # steps of a part's sum: n / 148 keys
    assert (np.abs(_np(out)[0] - want) <= want * (share + half * 1.01)).all()
    assert (np.abs(_np(lse)[0] - np.log(total)) <= share + 2.0 ** -23 * np.log(total)).all()
