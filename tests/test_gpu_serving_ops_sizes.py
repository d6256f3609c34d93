"""The batch-serving operators at the sizes that choose other forms of their kernels: large batches of few KV heads, long lists of
rows, many heads, long contexts.  Tolerances are those of the helpers in test_gpu_serving_ops."""
import numpy as np
import pytest

from tests.test_gpu_serving_ops import Batch

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


# ------------------------------------------------------------------ large batches whose KV heads fill no CTA
FEW = [  # requests, longest, kv_heads, group, dim, block, elem, dtype
    (700, 90, 1, 8, 128, 16, 1, "bfloat16"),     # four warps a head, whole
    (700, 900, 1, 3, 64, 16, 2, "float32"),      # ... and split
    (310, 500, 2, 8, 64, 5, 1, "float32"),
    (310, 800, 2, 4, 128, 16, 2, "bfloat16"),
    (310, 500, 3, 2, 128, 16, 1, "bfloat16"),    # a warp a head, one of four idle, whole
    (310, 800, 3, 2, 64, 16, 1, "float32"),
    (290, 512, 5, 2, 64, 16, 2, "bfloat16"),
    (290, 513, 5, 2, 64, 16, 1, "float32"),
    (200, 60, 2, 12, 64, 16, 1, "bfloat16"),     # two KV heads of two passes each: four units, a warp each
    (200, 60, 1, 20, 64, 16, 2, "float32"),      # ... of three passes
]


@pytest.mark.parametrize("case", FEW, ids=lambda c: "-".join(map(str, c)))
def test_attention_of_large_batches_over_few_kv_heads(kv, torch, case):
    n, top, hkv, group, d, block, elem, dtype = case
    lens = np.random.default_rng(n).integers(0, min(top, 120), n)
    lens[[0, n // 2]] = top, 0
    b = Batch(kv, torch, lens.tolist(), hkv, group, d, block, elem, getattr(torch, dtype))
    b.run(kv)
    b.check(torch)
