"""Batched attention where queries, keys and scores are very large or very small but every score is a number of fp32: results are those of
the definition, whatever lies between.

Keys are of size 2^a, queries of 2^b, so scores of 2^(a + b).  Where that is about 1, the bound of the batched attention's tests
(tests/test_gpu_serving_ops.py).  Where it is 2^20 and more, one key has all the weight: with A = scale * sum |q_i k_i|, a score is off by at
most A 2^-15 (the same bound's first part), so where the two largest are more than A 2^-13 apart (128 and more: the others weigh less
than 2^-180) the result is that key's value, off by 2^-14 of itself (the parts of a weight, the exponentials and factors that join warps and
parts) and its own rounding, and lse is its score, off by A 2^-13.
"""
import numpy as np
import pytest

from oracle import serving_oracle as S
from tests.test_gpu_serving_ops import Batch, _half_step, _np

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


PLACES = [  # lens, kv_heads, group, dim, block: whole contexts, split ones over pages that end inside a stage, a warp per KV head
    ([130, 0, 1, 33], 2, 4, 128, 16),
    ([640, 1100, 1], 3, 2, 64, 7),
    ([40] * 90 + [700], 8, 2, 128, 16),
]


@pytest.mark.parametrize("powers", [(40, -40), (97, -97), (-97, 97), (30, 0), (0, 30), (112, -60), (118, 0), (0, 118), (-97, 118)], ids=str)
@pytest.mark.parametrize("place", PLACES, ids=lambda p: f"{len(p[0])}x{max(p[0])}-{p[4]}")
@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_of_large_and_small_keys_and_queries(kv, torch, dtype, elem, place, powers):
    lens, hkv, group, d, block = place
    a, b = powers
    batch = Batch(kv, torch, lens, hkv, group, d, block, elem, getattr(torch, dtype), sizes=(a, a + 1), q_size=0.3 * 2.0 ** b)
    batch.run(kv)
    if a + b == 0:
        batch.check(torch)
        return
    q, out, lse, half = _np(batch.q), _np(batch.out), _np(batch.lse), _half_step(torch, batch.q.dtype)
    seen = 0
    for r, n in enumerate(lens):
        if n == 0:
            assert (out[r] == 0).all() and (lse[r] == -np.inf).all()
            continue
        for h in range(hkv * group):
            k, v = batch.k[r][:, h // group], batch.v[r][:, h // group]
            s, size = k @ q[r, h] * d ** -0.5, (np.abs(k) @ np.abs(q[r, h])).max() * d ** -0.5
            order = np.argsort(s)
            assert np.abs(s).max() < 2.0 ** 126
            if n > 1 and s[order[-1]] - s[order[-2]] <= size * 2.0 ** -13:
                continue
            seen += 1
            want = v[order[-1]]
            assert (np.abs(out[r, h] - want) <= np.abs(want) * (2.0 ** -14 + half * 1.01)).all(), (r, h, out[r, h] / want)
            assert abs(lse[r, h] - s[order[-1]]) <= size * 2.0 ** -13, (r, h, lse[r, h], s[order[-1]])
    assert seen > 0.8 * hkv * group * sum(n > 0 for n in lens)


@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("scale", [1e-37, 2.0 ** -20, 2.0 ** 30, 2.0 ** 100], ids=lambda x: f"{x:.0e}")
def test_attention_of_small_and_large_softmax_scales(kv, torch, dtype, elem, scale):
    """Queries of the size that the scale leaves for scores of about 1; of size 1 under the smallest scale, where all weights are alike."""
    batch = Batch(kv, torch, [200, 1, 900, 0, 17], 2, 4, 64, 16, elem, getattr(torch, dtype), q_size=0.03 / scale if scale > 1e-30 else 1.0)
    batch.run(kv, softmax_scale=scale)
    batch.check(torch, scale=scale)


@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("many", [False, True])
def test_attention_of_scores_that_the_scale_takes_out_of_fp32(kv, torch, dtype, elem, many):
    """Products that fp32 holds and scores that it does not: one above the range makes NaN of out and lse, those below it weigh nothing
    (also where a warp, or a part of the context, has no others), and a context of them alone is NaN."""
    lens, scale = [5, 5, 40, 1500, 300] + ([20] * 90 if many else []), 2.0 ** 40
    batch = Batch(kv, torch, lens, 8, 2, 64, 16, elem, getattr(torch, dtype), sizes=(-40, -39))
    batch.q.zero_()
    batch.q[..., 3] = torch.linspace(0.5, 1.5, 16).cuda().to(batch.q.dtype)
    gone = [[], [], [7], list(range(700)) + [1499], list(range(16, 300))]

    def put(r, at, size):
        pos = np.asarray(at)
        batch.k[r][pos] = 0
        batch.k[r][pos, :, 3] = size
        slots = torch.from_numpy(batch.table.cpu().numpy()[r, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
        rows = [torch.from_numpy(x[r][pos].astype(np.float32)).cuda() for x in (batch.k, batch.v)]
        kv.kv_op_cache_write(batch.cache, batch.layer, rows[0], rows[1], slots)
    put(0, [2], 2.0 ** 100)
    put(1, list(range(5)), -2.0 ** 100)
    for r, at in enumerate(gone):
        if at:
            put(r, at, -2.0 ** 100)
            batch.k[r], batch.v[r] = np.delete(batch.k[r], at, 0), np.delete(batch.v[r], at, 0)
    batch.run(kv, softmax_scale=scale)
    assert torch.isnan(batch.out[:2]).all() and torch.isnan(batch.lse[:2]).all()
    left = [n - (len(gone[r]) if r < len(gone) else 0) for r, n in enumerate(lens)]
    batch.check(torch, scale=scale, lens=left, only=range(2, len(lens)))
