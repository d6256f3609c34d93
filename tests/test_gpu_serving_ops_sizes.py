"""The batch-serving operators at the sizes that choose other forms of their kernels: large batches of few KV heads, long lists of
rows, many heads, long contexts.  Tolerances are those of the helpers in test_gpu_serving_ops."""
import numpy as np
import pytest

from oracle import serving_oracle as S
from tests.test_gpu_serving_ops import Batch, _half_step, _np, _pages_numpy, _rope_rows, _shape

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


# ------------------------------------------------------------------ long contexts
LONG = [  # lens, kv_heads, group, dim, block, elem, dtype
    ([5000], 1, 8, 128, 16, 2, "float32"),           # 79 records of a head: four warps go through them twice
    ([9001, 0, 77], 1, 3, 128, 16, 1, "bfloat16"),
    ([9001] + [3] * 24, 8, 8, 64, 16, 1, "float32"), # ... and one warp four times
    ([20011], 2, 4, 64, 16, 1, "float32"),
    ([20011, 5], 1, 9, 64, 24, 2, "bfloat16"),
    ([6000, 6001] + [9] * 400, 2, 2, 128, 16, 1, "bfloat16"),
]


@pytest.mark.parametrize("case", LONG, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}x{c[2]}-{c[3]}-{c[4]}-{c[5]}-{c[6]}")
def test_attention_of_long_contexts(kv, torch, case):
    lens, hkv, group, d, block, elem, dtype = case
    b = Batch(kv, torch, lens, hkv, group, d, block, elem, getattr(torch, dtype))
    b.run(kv)
    b.check(torch)


# ------------------------------------------------------------------ rows: two tokens to a thread, more heads than a CTA takes
def _quantised(x):
    """S.quantise_row of every row of finite values x [..., d] at once: (codes uint8, scale bytes)."""
    x = np.asarray(x, dtype=np.float64)
    most = np.abs(x).max(-1)
    part, power = np.frexp(most)                    # most = part 2^power, 1/2 <= part < 1; 448 = 0.875 2^9
    e = np.where(most > 0, np.clip(power - 9 + (part > 0.875), S.MIN_EXP, S.MAX_EXP), S.MIN_EXP)
    table = S.e4m3_values()[:127]
    y = np.minimum(np.abs(x) * 2.0 ** -e[..., None].astype(float), 448.0)
    hi = np.searchsorted(table, y).clip(0, 126)
    lo = np.maximum(hi - 1, 0)
    low, high = y - table[lo], table[hi] - y
    code = np.where((low < high) | ((low == high) & (lo % 2 == 0)), lo, hi)
    return np.where(np.signbit(x), code + 128, code).astype(np.uint8), (e + 127).astype(np.uint8)


ROWS = [  # tokens, kv_heads, dim, block
    (9473, 8, 64, 16), (4801, 8, 128, 16), (4737, 8, 128, 7),      # two tokens to a thread, an odd one at the end
    (41, 17, 128, 16), (37, 33, 64, 16), (2231, 17, 128, 16), (2305, 33, 64, 5),
    (5, 70, 128, 16),
]


@pytest.mark.parametrize("case", ROWS, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_rows_of_many_tokens_and_heads(kv, torch, case, elem, dtype):
    t, hkv, d, block = case
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(t)
    nb = -(-t // block) + 3
    cache = kv.PagedCache(_shape(hkv, d, block), nb, elem_bytes=elem)
    cache.data.view(torch.uint8).fill_(0x5A)
    want = _pages_numpy(cache).copy()[0]
    x = rng.standard_normal((2, t, hkv, d)).astype(np.float32) * 2.0 ** rng.integers(-30, 30, (2, t, hkv, 1)).astype(np.float32)
    both = torch.from_numpy(x).cuda().to(dtype)
    order = rng.permutation(nb * block)[:t].astype(np.int64)
    order[rng.random(t) < 0.1] = -1                               # padding in either place of a pair
    order[-1], order[0] = nb * block, order[0]
    slots = torch.from_numpy(order).cuda()
    k, v = both[0], both[1].transpose(0, 1).contiguous().transpose(0, 1)
    kv.kv_op_cache_write(cache, 0, k, v, slots)
    xs = both.float().cpu().numpy()
    live = (order >= 0) & (order < nb * block)
    blocks, offsets = order[live] // block, order[live] % block
    decoded = np.full((2, t, hkv, d), 7.0)
    values = block * hkv * d * elem
    for c in range(2):
        if elem == 1:
            codes, bytes_ = _quantised(xs[c])
            for i in (0, t // 2, t - 1):
                ref = S.quantise_row(xs[c, i, hkv - 1])
                assert np.array_equal(codes[i, hkv - 1], ref[0]) and bytes_[i, hkv - 1] == ref[1]
            page = want[c, :, :values].reshape(nb, block, hkv, d)
            page[blocks, offsets] = codes[live]
            scale = want[c, :, values:values + hkv * block].reshape(nb, hkv, block)
            scale[blocks, :, offsets] = bytes_[live]
            want[c, :, :values], want[c, :, values:values + hkv * block] = page.reshape(nb, -1), scale.reshape(nb, -1)
            decoded[c, live] = S.e4m3_values()[codes[live]] * 2.0 ** (bytes_[live].astype(float) - 127)[..., None]
        else:
            raw = torch.from_numpy(xs[c]).to(torch.bfloat16)
            page = want[c].reshape(nb, block, hkv, d * 2)
            page[blocks, offsets] = raw.view(torch.uint8).numpy().reshape(t, hkv, d * 2)[live]
            want[c] = page.reshape(nb, -1)
            decoded[c, live] = raw.double().numpy()[live]
    assert np.array_equal(_pages_numpy(cache)[0], want)
    for out_type in (torch.bfloat16, torch.float32):
        ko = torch.full((t, hkv, d), 7.0, dtype=out_type, device="cuda")
        vo = torch.full((hkv, t, d), 7.0, dtype=out_type, device="cuda").transpose(0, 1)
        kv.kv_op_cache_read(cache, 0, slots, ko, vo)
        assert np.array_equal(_np(ko), decoded[0]) and np.array_equal(_np(vo), decoded[1])


# ------------------------------------------------------------------ rotary positions: two tokens to a CTA, the last one alone
TURNS = [  # tokens, heads, head_dim, rotary, layout, dtype, arrangement
    (2501, 3, 64, 64, "interleaved", "bfloat16", "plain"),
    (1187, 9, 128, 128, "half", "bfloat16", "qkv"),
    (1187, 3, 64, 32, "half", "float32", "heads"),
    (1187, 9, 128, 102, "half", "bfloat16", "qkv"),            # whole rows through shared memory
    (1185, 5, 64, 50, "half", "float32", "plain"),
    (1187, 2, 64, 64, "half", "bfloat16", "odd"),              # rows that start on no vector
    (1185, 3, 65, 40, "interleaved", "float32", "plain"),
]


@pytest.mark.parametrize("case", TURNS, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope_of_an_odd_number_of_tokens(kv, torch, case, backward, in_place):
    t, h, d, rotary, layout, dtype, arrangement = case
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(5)
    x = _rope_rows(torch, t, h, d, dtype, arrangement, gen)
    pos = torch.randint(-70000, 70000, (t,), generator=gen, device="cuda").to(torch.int32)
    rope = kv.Rope(rotary, layout=layout, base=1e6, gain=1.1)
    xs, half = _np(x), rotary // 2
    guard = torch.full((t + 1, h, d + 16), 7.0, dtype=dtype, device="cuda")
    out = x if in_place else guard[:t, :, 8:8 + d]
    kv.kv_op_rope(rope, x, pos, out, backward=backward)
    first = np.arange(half) if layout == "half" else 2 * np.arange(half)
    second = first + half if layout == "half" else first + 1
    ang = pos.cpu().numpy().astype(float)[:, None] * rope.frequencies() * (-1 if backward else 1)
    cos, sin = 1.1 * np.cos(ang)[:, None], 1.1 * np.sin(ang)[:, None]
    want, size = xs.copy(), np.zeros_like(xs)
    a, b = xs[..., first], xs[..., second]
    want[..., first], want[..., second] = a * cos - b * sin, b * cos + a * sin
    size[..., first] = size[..., second] = np.abs(a) + np.abs(b)
    # as in test_gpu_serving_ops: angle 8e-7, six roundings of 2^-24, the result's
    tol = 1.1 * size * (8e-7 + 6 * 2.0 ** -24) + _half_step(torch, dtype) * np.abs(want)
    got = _np(out)
    assert np.array_equal(got[..., rotary:], xs[..., rotary:])
    assert (np.abs(got - want)[..., :rotary] <= tol[..., :rotary] * (1 + 2.0 ** -10)).all()
    if not in_place:
        assert (guard[:t, :, :8] == 7).all() and (guard[:t, :, 8 + d:] == 7).all() and (guard[t] == 7).all()
