"""What the parts of queries and weights leave of fp32 over e2m1 pages, seen one weight at a time (the way of
tests/test_gpu_serving_ops_precision.py, whose bounds these are).

Two fp16 parts: a weight is off by uw = 2^-22 of itself in calls of either type, an fp32 query by uq = 2^-22 (a bf16 query is one part, exact), and
a weight by 2^-36 of the request's largest contribution (a stored value is up to 2,688 times its row's power of two, and less than half of
that only where another row's is larger: twice the largest value times the largest weight).  The running maximum of the contributions may
be replaced twice (scores within 2 T < 8, values within a binade): a factor, 2^-22 and a rounding, each time.  The result's own rounding is
counted as what it is, half a unit in the last place of the result.

Sums over long contexts, fp32 calls: a warp adds the products of 16 keys at a time, N = n / 16 additions of positive numbers or fewer, each
rounded to nearest.  Such roundings have no sign in common, so over the results of a whole batch they add up as a random walk does: with a
sum that grows evenly, 2^-24 sqrt(N) / 3 of its size (a uniform error of half a unit, 1 / sqrt 3; steps that grow, another 1 / sqrt 3), and
the sums of the weights likewise.  Allowed, of the norm of the results: three times 2^-24 sqrt(N) and 2^-22 for the exponential.  Accumulated inside the matrix
instruction, which truncates, N additions of three or two parts lose N 2^-24 / 2 and more of the sum, all in one direction: several times that.
"""
import numpy as np
import pytest

from tests.test_gpu_serving_ops import _np, _shape
from tests.test_gpu_serving_ops_precision import PLACES

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


def _half_unit(torch, x, dtype):
    """Half a unit in the last place of numbers up to |x|."""
    return np.exp2(np.floor(np.log2(np.maximum(x, 2.0 ** -120)))) * torch.finfo(dtype).eps / 2


@pytest.mark.parametrize("top", [0.5, 3.5])
@pytest.mark.parametrize("place", PLACES, ids=lambda p: f"{len(p[0])}x{max(p[0])}")
@pytest.mark.parametrize("dim,block", [(64, 16), (128, 16), (128, 7)])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_one_weight_at_a_time(kv, torch, dtype, dim, block, place, top):
    lens, hkv, group, joins = place
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(dim + block)
    hq, need = hkv * group, [-(-n // block) for n in lens]
    cache = kv.PagedCache(_shape(hkv, dim, block), sum(need), elem_bytes=0.5, fill=0)
    table = np.full((len(lens), max(need)), -1, dtype=np.int32)
    order, at = rng.permutation(sum(need)), 0
    keys, values = [], []
    for r, n in enumerate(lens):
        table[r, :need[r]] = order[at:at + need[r]]
        at += need[r]
        k, v = rng.uniform(-1, 1, (n, hkv, dim)).astype(np.float32), np.zeros((n, hkv, dim), np.float32)
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
    size = rng.uniform(0.7, 1.0, (len(lens), hq)) * top / scale / np.log2(np.e) / 1.125      # a code of 6 and a scale round to at most 1.125
    np.put_along_axis(q, which[..., None], size[..., None], -1)
    q = torch.from_numpy(q).cuda().to(dtype)
    out, lse = torch.empty_like(q), torch.empty(len(lens), hq, device="cuda")
    ctx = max(lens)
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(len(lens), hq, cache, ctx), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, torch.from_numpy(table).cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), ctx,
                                     out, scratch, lse=lse, softmax_scale=scale)
    qs, got, got_lse = _np(q), _np(out), _np(lse)
    uq, uw = 0.0 if dtype is torch.bfloat16 else 2.0 ** -22, 2.0 ** -22
    factor = 2.0 ** -22 + 2.0 ** -24
    for r, n in enumerate(lens):
        for h in range(hq):
            g = h // group
            s = keys[r][:, g, which[r, h]] * qs[r, h, which[r, h]] * scale
            t = np.abs(s).max() * np.log2(np.e)
            assert t < 4
            p = np.exp(s)
            want = p @ values[r][:, g] / p.sum()
            score = t * (uq + 10 * 2.0 ** -24) + 2.0 ** -22
            sums = score + (n / 8 + 16) * 2.0 ** -24 + joins * factor
            share = score + uw + (joins + 2) * factor + sums + factor
            off = np.abs(want) * share * (1 + 2.0 ** -8) + 2.0 ** -36 * 2 * 1.875 * p.max() / p.sum()
            tol = off + _half_unit(torch, np.abs(want) + off, dtype)
            err = np.abs(got[r, h] - want)
            assert (err <= tol).all(), (r, h, n, (err / tol).max(), share)
            lse_want = np.log(p.sum())
            assert abs(got_lse[r, h] - lse_want) <= sums + 2.0 ** -21 + 2.0 ** -22 * abs(lse_want), (r, h, got_lse[r, h], lse_want)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("elem", [0.5, 2])
def test_sums_over_a_long_context_do_not_drift(kv, torch, elem, dim):
    n, requests, heads, block = 16384, 128, 8, 16
    rng = np.random.default_rng(dim)
    cache = kv.PagedCache(_shape(heads, dim, block), n // block, elem_bytes=elem)
    rows = [torch.from_numpy(x.astype(np.float32)).cuda() for x in (rng.uniform(-1, 1, (n, heads, dim)), rng.uniform(0.5, 3, (n, heads, dim)))]
    slots = torch.arange(n, device="cuda")
    kv.kv_op_cache_write(cache, 0, rows[0], rows[1], slots)
    kv.kv_op_cache_read(cache, 0, slots, rows[0], rows[1])
    q = torch.from_numpy(rng.uniform(-0.5, 0.5, (requests, heads, dim)).astype(np.float32)).cuda()
    out = torch.empty_like(q)
    table = torch.arange(n // block, dtype=torch.int32, device="cuda").expand(requests, -1).contiguous()      # one context, attended to by all
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(requests, heads, cache, n), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, table, torch.full((requests,), n, dtype=torch.int32, device="cuda"), n, out, scratch)
    k, v, q = (x.double() for x in (*rows, q))
    p = torch.softmax(torch.einsum("rhd,nhd->rhn", q, k) * dim ** -0.5, -1)
    want = torch.einsum("rhn,nhd->rhd", p, v)
    assert float((out.double() - want).norm() / want.norm()) <= 3 * 2.0 ** -24 * (n / 16) ** 0.5 + 2.0 ** -22
