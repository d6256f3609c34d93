"""What the 16-bit parts of queries and weights leave of fp32, seen one weight at a time.

A head's query has one value that is not 0, a key's value row one too, and each in a dim of its own: a score is one product and a
dim of the result one weight, so nothing is summed but zeros and the bounds are those of the parts themselves, far below what
sums over whole rows have to allow.

Bounds.  Scores in base 2, t = s log2(e), |t| <= T.  A query is off by uq of itself: 0 in bf16 calls (one part), 2^-24 over bf16 pages (three
bf16) and 2^-22 over e4m3 pages (two fp16) in fp32 calls.  Up to 10 roundings of 2^-24 of T follow: the sums of the parts, the scale (to
fp32, its product with log2(e), that constant, the product with the score), and t - m (|t| + |m| <= 2 T).  2^t is off by 2^-22 more, a weight
by uw: 2^-24 (three bf16), 2^-22 (two fp16), in bf16 calls over bf16 pages 2^-16 (two bf16).  So a weight is off by
  w = T (uq + 10 2^-24) + 2^-22 + uw   (ln 2 < 1 is left in the first term)
and in the sum of the weights, which takes them whole, by the same without uw; its additions: n / 8 + 16 of 2^-24.  Factors that join the
warps of a CTA, the parts and the warps that join the parts: up to 4, each 2^-22 and a rounding, on both sides; the division 2^-22, the
result's rounding half a step.  T stays below 4, so that the running maximum is set once.
"""
import numpy as np
import pytest

from tests.test_gpu_serving_ops import _half_step, _np, _shape

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


PLACES = [  # lens, kv_heads, group, factors that join: whole contexts, split ones, a warp per KV head
    ([100, 37], 2, 4, 1),
    ([900, 37], 2, 8, 4),
    ([90] * 80, 8, 2, 0),
    ([90] * 79 + [900], 8, 2, 2),
]


@pytest.mark.parametrize("top", [0.5, 3.5])
@pytest.mark.parametrize("place", PLACES, ids=lambda p: f"{len(p[0])}x{max(p[0])}")
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_one_weight_at_a_time(kv, torch, dtype, elem, dim, place, top):
    lens, hkv, group, joins = place
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(dim + elem)
    block, hq = 16, hkv * group
    need = [-(-n // block) for n in lens]
    cache = kv.PagedCache(_shape(hkv, dim, block), sum(need), elem_bytes=elem)
    table = np.full((len(lens), max(need)), -1, dtype=np.int32)
    order, at = rng.permutation(sum(need)), 0
    keys, values = [], []
    for r, n in enumerate(lens):
        table[r, :need[r]] = order[at:at + need[r]]
        at += need[r]
        # the key's values in [-1, 1] x at least 1 once, so that an e4m3 row keeps its scale
        k = rng.uniform(-1, 1, (n, hkv, dim)).astype(np.float32)
        v = np.zeros((n, hkv, dim), np.float32)
        for g in range(hkv):
            some = rng.permutation(n)[:dim]
            v[some, g, rng.permutation(dim)[:len(some)]] = rng.choice([1.0, -1.25, 1.5, 1.875], len(some))
        pos = np.arange(n)
        slots = torch.from_numpy(table[r, pos // block].astype(np.int64) * block + pos % block).cuda()
        kv.kv_op_cache_write(cache, 0, torch.from_numpy(k).cuda(), torch.from_numpy(v).cuda(), slots)
        back = torch.empty(2, n, hkv, dim, device="cuda")
        kv.kv_op_cache_read(cache, 0, slots, back[0], back[1])
        keys.append(_np(back[0]))
        values.append(_np(back[1]))
    scale = 0.125
    q = np.zeros((len(lens), hq, dim))
    which = rng.integers(0, dim, (len(lens), hq))
    size = rng.uniform(0.7, 1.0, (len(lens), hq)) * top / scale / np.log2(np.e) / 1.0625      # keys round to at most 1.0625
    np.put_along_axis(q, which[..., None], size[..., None], -1)
    q = torch.from_numpy(q).cuda().to(dtype)
    out, lse = torch.empty_like(q), torch.empty(len(lens), hq, device="cuda")
    ctx = max(lens)
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(len(lens), hq, cache, ctx), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, torch.from_numpy(table).cuda(),
                                     torch.tensor(lens, dtype=torch.int32, device="cuda"), ctx, out, scratch, lse=lse,
                                     softmax_scale=scale)
    qs, got, got_lse, half = _np(q), _np(out), _np(lse), _half_step(torch, dtype)
    uq = 0.0 if dtype is torch.bfloat16 else (2.0 ** -22 if elem == 1 else 2.0 ** -24)
    uw = 2.0 ** -22 if elem == 1 else (2.0 ** -16 if dtype is torch.bfloat16 else 2.0 ** -24)
    worst = 0.0
    for r, n in enumerate(lens):
        for h in range(hq):
            g = h // group
            s = keys[r][:, g, which[r, h]] * qs[r, h, which[r, h]] * scale
            t = np.abs(s).max() * np.log2(np.e)
            assert t < 4
            p = np.exp(s)
            want = p @ values[r][:, g] / p.sum()
            score = t * (uq + 10 * 2.0 ** -24) + 2.0 ** -22
            sums = score + (n / 8 + 16) * 2.0 ** -24 + joins * (2.0 ** -22 + 2.0 ** -24)
            share = score + uw + joins * (2.0 ** -22 + 2.0 ** -24) + sums + 2.0 ** -22 + 2.0 ** -24
            tol = np.abs(want) * (share + half) * (1 + 2.0 ** -8)
            if elem == 1:
                tol = tol + 2.0 ** -36 * 2 * 1.875 * p.max() / p.sum()      # a weight's floor, twice where a maximum is 1 off
            err = np.abs(got[r, h] - want)
            worst = max(worst, (err / np.maximum(tol, 1e-30)).max())
            assert (err <= tol).all(), (r, h, n, (err / np.maximum(np.abs(want), 1e-30)).max(), share)
            lse_want = np.log(p.sum())
            assert abs(got_lse[r, h] - lse_want) <= sums + 2.0 ** -21 + 2.0 ** -22 * abs(lse_want), (r, h, got_lse[r, h], lse_want)
    print("largest share of a bound:", worst)
