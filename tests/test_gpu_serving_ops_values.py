"""The batch-serving operators at values where arithmetic can go wrong: infinities and NaN inside contexts and queries, scores
that leave fp32."""
import math

import numpy as np
import pytest

from oracle import serving_oracle as S
from tests.test_gpu_serving_ops import Batch, _np, _shape

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


# ------------------------------------------------------------------ infinities and NaN
def _rewrite(kv, torch, b, r, pos, k=None, v=None):
    """Puts the rows k and v [kv_heads, dim] (default: what is there) at position pos of request r."""
    block = b.cache.block_size
    slot = torch.tensor([int(b.table[r, pos // block]) * block + pos % block], device="cuda")
    rows = [b.k[r][pos] if k is None else k, b.v[r][pos] if v is None else v]
    rows = [torch.from_numpy(np.asarray(x, dtype=np.float32)).cuda()[None] for x in rows]
    kv.kv_op_cache_write(b.cache, b.layer, rows[0], rows[1], slot)


PLACES = [  # lens, kv_heads, group, dim, block, request, position: whole contexts, split ones, a warp per KV head
    ([70, 0, 33], 2, 4, 128, 16, 0, 41),
    ([33, 640, 1000], 2, 4, 64, 16, 1, 639),
    ([700, 2600], 3, 12, 128, 7, 1, 0),
    ([40] * 90 + [300], 8, 2, 64, 16, 90, 170),
    ([40] * 90 + [700], 8, 4, 128, 16, 90, 355),
]


@pytest.mark.parametrize("place", PLACES, ids=lambda p: f"{len(p[0])}x{max(p[0])}-{p[1]}x{p[2]}-{p[3]}")
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan], ids=str)
def test_attention_infinities_and_nan_reach_what_they_enter(kv, torch, place, elem, dtype, value):
    """A query's: its head.  A key's: the group's heads and their lse.  A value's: its dim of the group's heads.  All else is what
    it is without them."""
    lens, hkv, group, d, block, r, pos = place
    b = Batch(kv, torch, lens, hkv, group, d, block, elem, getattr(torch, dtype))
    dim, g = 11, hkv - 1
    heads = slice(g * group, (g + 1) * group)
    b.q[:, :, dim] = 0.3                             # no product of the key's infinity is zero, and all have one sign
    b.run(kv)
    b.check(torch)
    out, lse = b.out.clone(), b.lse.clone()

    def differs(o_nan, l_nan):
        b.scratch.fill_(0xFF)
        b.out.fill_(7)
        b.run(kv)
        assert torch.equal(torch.isnan(b.out), o_nan) and torch.equal(torch.isnan(b.lse), l_nan)
        assert torch.equal(b.lse[~l_nan], lse[~l_nan]) and torch.equal(b.out[~o_nan], out[~o_nan])

    none_o, none_l = torch.zeros_like(out, dtype=torch.bool), torch.zeros_like(lse, dtype=torch.bool)
    b.q[r, 1, dim] = value
    o_nan, l_nan = none_o.clone(), none_l.clone()
    o_nan[r, 1], l_nan[r, 1] = True, True
    differs(o_nan, l_nan)
    b.q[r, 1, dim] = 0.3

    k, v = b.k[r][pos].copy(), b.v[r][pos].copy()
    low = np.abs(v[g]).argmin()                      # e4m3: the row's scale is that of its finite values
    low = dim if low == dim or elem == 2 else low
    v[g, low] = value
    _rewrite(kv, torch, b, r, pos, v=v)
    o_nan, l_nan = none_o.clone(), none_l.clone()
    o_nan[r, heads, low] = True
    differs(o_nan, l_nan)

    k[g, dim] = value
    _rewrite(kv, torch, b, r, pos, k=k)
    o_nan, l_nan = none_o.clone(), none_l.clone()
    o_nan[r, heads], l_nan[r, heads] = True, True
    differs(o_nan, l_nan)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("lens", [[50, 9], [900, 9], [900, 9] + [3] * 120], ids=lambda x: f"{len(x)}x{x[0]}")
def test_attention_scores_below_fp32_weigh_nothing(kv, torch, lens, dtype):
    """Keys of the type's lowest value: q . k is below fp32's range.  In exact arithmetic their weight is 0 (to far more than 64
    bits), so the result is that of the other keys."""
    b = Batch(kv, torch, lens, 8, 2, 128, 16, 2, getattr(torch, dtype))
    b.q.abs_()
    b.q += 0.05
    gone = [0, 17, lens[0] - 1]
    for pos in gone:
        _rewrite(kv, torch, b, 0, pos, k=np.full((8, 128), torch.finfo(torch.bfloat16).min))
    for x in (b.k, b.v):
        x[0] = np.delete(x[0], gone, axis=0)
    b.run(kv)
    b.check(torch, lens=[lens[0] - 3] + lens[1:])


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("n", [5, 1500])
def test_attention_of_no_score_that_is_a_number(kv, torch, n, dtype):
    """Every score below fp32's range: nothing is left to divide by, and lse says so as well."""
    b = Batch(kv, torch, [n, 20], 2, 2, 64, 16, 2, getattr(torch, dtype))
    b.q.abs_()
    b.q += 0.05
    for pos in range(n):
        b.k[0][pos] = torch.finfo(torch.bfloat16).min
    pos = torch.arange(n, device="cuda")
    slots = b.table[0].long()[pos // 16] * 16 + pos % 16
    kv.kv_op_cache_write(b.cache, 0, torch.from_numpy(b.k[0]).float().cuda(), torch.from_numpy(b.v[0]).float().cuda(), slots)
    b.run(kv)
    assert torch.isnan(b.out[0]).all() and torch.isnan(b.lse[0]).all()
    b.check(torch, only=[1])


# ------------------------------------------------------------------ small weights beside a large one
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_many_small_weights_beside_a_large_one(kv, torch, dtype):
    """e4m3 pages: one key with e^23 times the weight of each of the others, whose values lie in a dim where its own is 0.  There are
    so many KV heads that one part holds the context.  A weight may be off by 2^-36 of the largest contribution (1 here) and
    2^-22 of itself, sums and the factors that join them by (n / 16 + 64) 2^-22 of what they hold."""
    n, one, heads = 16384, 777, 300
    cache = kv.PagedCache(_shape(heads, 64, 16), n // 16, elem_bytes=1)
    k, v = torch.zeros(n, 1, 64, device="cuda"), torch.zeros(n, 1, 64, device="cuda")
    k[one, :, 0], v[one, :, 0] = 1.0, 1.0
    v[:, :, 1] = 1.0
    v[one, :, 1] = 0.0
    kv.kv_op_cache_write(cache, 0, k.expand(n, heads, 64), v.expand(n, heads, 64), torch.arange(n, device="cuda"))
    q = torch.zeros(1, heads, 64, dtype=getattr(torch, dtype), device="cuda")
    q[:, :, 0] = 23.0
    out, table = torch.empty_like(q), torch.arange(n // 16, dtype=torch.int32, device="cuda")[None]
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(1, heads, cache, n), dtype=torch.uint8, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, table, lens, n, out, scratch, softmax_scale=1.0)
    small = (n - 1) * math.exp(-23.0)
    want0, want1 = 1 / (1 + small), small / (1 + small)
    got = _np(out)[0]
    # 23 is exact in both types, so are the scores; the exponent of a weight is rounded to 2^-24 of 23 log2(e) = 33: 2^-19
    share = 2.0 ** -18 + 2.0 ** -21 + (n / 16 + 64) * 2.0 ** -22 + torch.finfo(q.dtype).eps
    assert (np.abs(got[:, 1] - want1) <= n * 2.0 ** -36 + want1 * share).all(), (got[:, 1], want1)
    assert (np.abs(got[:, 0] - want0) <= want0 * share).all(), (got[:, 0], want0)
    assert (got[:, 2:] == 0).all()
