"""Selections of batches whose contexts have thousands of blocks: how many CTAs share a line of blocks depends on the lines and on the
blocks' number, the choice does not.  Equal to the definition, in whole numbers; bounds are given, not formed."""
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


@pytest.mark.parametrize("requests,heads", [(1, 8), (4, 8), (9, 8), (75, 2), (160, 1)])
@pytest.mark.parametrize("blocks", [700, 5_700, 5_900, 9_001])
def test_select_in_batches_of_long_contexts(kv, torch, requests, heads, blocks):
    d, block, keep, first, last, group = 64, 16, 40, 1, 2, 2
    rng = np.random.default_rng(blocks + requests)
    pool = 10_000
    cache = kv.PagedCache(_shape(heads, d, 1), 1, elem_bytes=2)
    cache.num_blocks, cache.block_size = pool, block                        # bounds of a pool of keys that nothing reads
    bounds = kv.BlockBounds(cache)
    codes = rng.integers(-127, 128, (pool, heads, 2, d)).astype(np.int8)
    scales = rng.integers(118, 122, (pool, heads)).astype(np.uint8)
    bounds.codes[0].copy_(torch.from_numpy(codes))
    bounds.scales[0].copy_(torch.from_numpy(scales))
    lens = rng.integers(1, blocks * block + 1, requests)
    lens[0] = blocks * block
    table = rng.integers(0, pool, (requests, blocks)).astype(np.int32)
    q = torch.from_numpy(rng.standard_normal((requests, heads * group, d)).astype(np.float32)).cuda()
    kept = torch.full((requests, heads, keep), 777, dtype=torch.int32, device="cuda")
    kept_lens = torch.empty(requests, dtype=torch.int32, device="cuda")
    scratch = torch.empty(kv.kv_select_blocks_scratch_bytes(requests, bounds, blocks * block), dtype=torch.uint8, device="cuda")
    kv.kv_op_select_blocks(q, bounds, 0, torch.from_numpy(table).cuda(), torch.from_numpy(lens.astype(np.int32)).cuda(), blocks * block,
                           kept, kept_lens, scratch, first=first, last=last)
    got, qs = kept.cpu().numpy(), _np(q)
    for r in range(requests):
        n = -(-int(lens[r]) // block)
        assert int(kept_lens[r]) == lens[r] - max(n - keep, 0) * block
        for h in range(heads):
            if n <= keep:
                assert np.array_equal(got[r, h], np.concatenate([table[r, :n], np.full(keep - n, -1)]))
                continue
            # every number below 2^31 is exact in fp64, and so are sums of them below 2^53
            mid = np.arange(first, n - last)
            rows = table[r, mid]
            whole = codes[rows, h].reshape(len(mid), -1).astype(np.float64) @ P.query_code(qs[r, h * group:(h + 1) * group]).astype(np.float64)
            score = whole.astype(np.float32) * 2.0 ** (scales[rows, h].astype(np.float64) - 127)
            best = mid[np.lexsort((mid, -score))[:keep - first - last]]
            want = np.sort(np.concatenate([np.arange(first), best, np.arange(n - last, n)]))
            assert np.array_equal(got[r, h], table[r, want]), (r, h, n)
