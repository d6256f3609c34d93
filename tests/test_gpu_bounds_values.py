"""Bounds of blocks whose keys are near zero: largest values rounded up, smallest rounded down, subnormal ones among them.  Whole numbers,
equal to the oracle's (oracle/pages4_oracle.py)."""
import numpy as np
import pytest

from oracle import pages4_oracle as P
from tests.test_gpu_serving_ops import _shape

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


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [1, 16, 48])
def test_bounds_of_subnormal_keys(kv, torch, d, block):
    rng = np.random.default_rng(d + block)
    nb, heads = 7, 3
    bits = np.zeros((nb, block, heads, d), np.uint16)                     # bf16 patterns
    bits[0] = rng.integers(1, 0x80, bits[0].shape)                         # subnormal, positive
    bits[1] = rng.integers(0x8001, 0x8080, bits[1].shape)                  # ... negative
    bits[2] = rng.integers(0, 0x80, bits[2].shape) | rng.integers(0, 2, bits[2].shape) << 15      # both, and zeros of both signs
    bits[3], bits[3, 0, :, 5] = bits[2], 0x42FE                            # ... beside a key of 127: the unit is 1
    bits[4], bits[4, 0, :, 5] = bits[2], 0xC2FF                            # ... of -127.5: the unit is 2
    bits[5, 0, :, ::2], bits[5, 0, :, 1::2] = 1, 0x8001                    # the smallest there are
    bits[6] = rng.integers(0x80, 0x2180, bits[6].shape)                    # the smallest normal ones up to the bound's least unit
    cache = kv.PagedCache(_shape(heads, d, block), nb)
    cache.data[0, 0] = torch.from_numpy(bits.reshape(nb, -1).view(np.int16)).cuda()
    bounds = kv.BlockBounds(cache)
    blocks = torch.arange(nb, dtype=torch.int32, device="cuda")
    kv.kv_op_block_bounds(cache, 0, blocks, torch.full((nb,), block, dtype=torch.int32, device="cuda"), bounds)
    codes, scales = bounds.codes.cpu().numpy()[0], bounds.scales.cpu().numpy()[0]
    keys = (bits.astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    for b in range(nb):
        for h in range(heads):
            want, byte = P.block_bounds(keys[b, :, h])
            assert scales[b, h] == byte and np.array_equal(codes[b, h], want), (b, h)
