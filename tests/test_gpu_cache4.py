"""A cache held in four bits on the GPU: e2m1 pages written, read, attended to and moved, and keys appended with their rotation, against
the fp64 oracle (oracle/pages4_oracle.py, oracle/serving_oracle.py).

Tolerances.  Pages: exact, every byte.  Appending: the bits of the rotary operator followed by the write of rows; the queries within the
bound of the rotary tests.  Attention: the bound of the batched attention's tests (tests/test_gpu_serving_ops.py): what it counts
for fp16 parts holds for every format whose values fp16 holds exactly, as it does code * scale of e2m1 pages (six bits,
2^-10 to 2688).
"""
import math

import numpy as np
import pytest

from oracle import pages4_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_serving_ops import ATTEND, LENGTHS, Batch, _half_step, _np, _pages_numpy, _shape

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


# ------------------------------------------------------------------ rows into pages and back
def _special_rows(d):
    """Rows at the borders of the format."""
    rng = np.random.default_rng(11)
    base = rng.standard_normal(d).astype(np.float32)
    rows = [base * 0, base, -base, np.where(np.arange(d) % 32 < 16, base, base * np.float32(2.0 ** -14))]
    for top in (2688.0, 2700.0, 2687.0, 6.0, 6.05, 5.95, 2.0 ** -100, 3.0e38, 2.0 ** -126, 1e-40, 3.3895e38, 1.3125 * 2.0 ** 60):
        r = base / 8
        r = np.where(np.abs(r) >= 1, 0.5, r).astype(np.float32) * np.float32(min(top, 1e30))
        r[3] = top
        rows.append(r)
    r = base.copy(); r[0] = np.inf; r[5] = -np.inf; r[17] = np.nan      # two groups of NaN, the others whole
    rows.append(r)
    r = base.copy(); r[d - 1] = -np.inf
    rows.append(r)
    rows.append(np.full(d, np.nan, np.float32))
    rows.append(np.full(d, -np.inf, np.float32))
    r = (np.arange(d) % 25).astype(np.float32) * 0.25 - 3; r[::16] = 6      # halves between codes of a group of scale 1, both signs
    rows.append(r)
    r = np.tile(np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0], np.float32), d // 8)      # ... of scales that are no powers of two
    rows.append(r * np.float32(1.375))
    rows.append(-r * np.float32(1.875 * 2.0 ** -7))
    rows.append(np.nextafter(r, np.float32(0)) * np.float32(1.125))        # just below them
    rows.append(np.nextafter(r * np.float32(1.625), np.float32(9)))       # just above
    r = np.zeros(d, np.float32); r[::2] = -0.0; r[1] = 448
    rows.append(r)
    r = base.copy(); r[0] = 2688 * 2.0 ** 9; r[16:] *= np.float32(2.0 ** -3)      # groups below the least scale
    rows.append(r)
    return np.stack(rows).astype(np.float32)


WRITE = [  # tokens, kv_heads, dim, block, layers, layout
    (1, 1, 64, 16, 1, "layer_major"), (5, 8, 128, 16, 2, "layer_major"), (67, 3, 64, 7, 2, "block_major"),
    (133, 2, 128, 32, 1, "layer_major"), (40, 8, 64, 1, 3, "block_major"), (90, 5, 128, 24, 1, "layer_major"),
]


@pytest.mark.parametrize("case", WRITE, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_write_then_read(kv, torch, case, dtype):
    t, hkv, d, block, layers, layout = case
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(t)
    nb = -(-t // block) + 3
    cache = kv.PagedCache(_shape(hkv, d, block, layers), nb, layout=layout, elem_bytes=0.5)
    assert cache.page_bytes == kv.kv_cache_page_bytes(block, hkv, d, 0.5)
    cache.data.fill_(0x5A)
    before = _pages_numpy(cache).copy()
    x = rng.standard_normal((2, t, hkv, d)).astype(np.float32) * 2.0 ** rng.integers(-30, 30, (2, t, hkv, 1)).astype(np.float32)
    special = _special_rows(d)
    for i in range(min(2 * t * hkv, len(special))):
        x[i % 2, i // 2 // hkv, i // 2 % hkv] = special[i]
    both = torch.from_numpy(x).cuda().to(dtype)
    slots = torch.from_numpy(rng.permutation(nb * block)[:t].astype(np.int64)).cuda()
    if t > 44:
        slots[42], slots[44] = -1, nb * block          # padding and a slot behind the pool: left out
    layer = layers - 1
    wide = torch.zeros(t, 3 * hkv, d, dtype=dtype, device="cuda")      # K out of a wide buffer, V head-major
    wide[:, hkv:2 * hkv] = both[0]
    k, v = wide[:, hkv:2 * hkv], both[1].transpose(0, 1).contiguous().transpose(0, 1)
    kv.kv_op_cache_write(cache, layer, k, v, slots)
    want = before.copy()
    records = want[layer].reshape(2, nb, hkv, -1)
    xs = both.float().cpu().numpy()
    decoded = np.zeros((2, t, hkv, d))
    for i, s in enumerate(slots.cpu().tolist()):
        for h in range(hkv):
            for c in range(2):
                codes, groups, byte = P.quantise_row(xs[c, i, h])
                decoded[c, i, h] = P.decode_row(codes, groups, byte)
                if not 0 <= s < nb * block:
                    continue
                b, o = divmod(s, block)
                rec = records[c, b, h]
                rec[o * d // 2:(o + 1) * d // 2] = codes[0::2] | codes[1::2] << 4
                at = block * d // 2 + o * (d // 16)
                rec[at:at + d // 16] = groups
                rec[block * (d // 2 + d // 16) + o] = byte
    assert np.array_equal(_pages_numpy(cache), want)
    # and back: exact in both types, rows without a slot untouched, slots repeated
    for out_type in (torch.bfloat16, torch.float32):
        again = torch.cat([slots, slots[:1]])
        ko = torch.full((t + 1, hkv, d), 7.0, dtype=out_type, device="cuda")
        vo = torch.full((hkv, t + 1, d), 7.0, dtype=out_type, device="cuda").transpose(0, 1)
        kv.kv_op_cache_read(cache, layer, again, ko, vo)
        for c, o in enumerate((ko, vo)):
            got = _np(o)
            for i, s in enumerate(again.cpu().tolist()):
                w = decoded[c, i % t] if 0 <= s < nb * block else np.full((hkv, d), 7.0)
                assert np.array_equal(got[i], w, equal_nan=True), (c, i, s)


def test_many_rows_and_every_code(kv, torch):
    """Rows enough for two tokens to a thread; pages of every code and scale read back as the values they stand for."""
    t, hkv, d = 5000, 8, 128
    cache = kv.PagedCache(_shape(hkv, d, 16), 320, elem_bytes=0.5)
    cache.data.copy_(torch.randint(0, 256, cache.data.shape, device="cuda", dtype=torch.uint8))
    rec = cache.data.view(2, 320, hkv, -1)
    rec[..., 16 * 72:16 * 73] = rec[..., 16 * 72:16 * 73] % 200 + 20
    slots = torch.randperm(320 * 16, device="cuda")[:t]
    k, v = torch.empty(2, t, hkv, d, device="cuda")
    kv.kv_op_cache_read(cache, 0, slots, k, v)
    codes = rec[..., :16 * 64].unflatten(-1, (16, 64))
    codes = torch.stack([codes & 15, codes >> 4], -1).flatten(-2).long()
    scale = torch.from_numpy(S.e4m3_values()).cuda()[rec[..., 16 * 64:16 * 72].long()].unflatten(-1, (16, 8)).repeat_interleave(16, -1)
    power = torch.exp2(rec[..., 16 * 72:16 * 73].double() - 127).unsqueeze(-1)
    want = torch.from_numpy(P.e2m1_values()).cuda()[codes] * scale * power          # [2, blocks, heads, 16, d]
    want = want.transpose(2, 3).flatten(1, 2)[:, slots]
    for got, w in ((k, want[0]), (v, want[1])):
        assert torch.equal(torch.isnan(got), torch.isnan(w)) and torch.equal(got.double().nan_to_num(7e77), w.nan_to_num(7e77))
    # written back, every row is what it was: its codes may take another scale, its values do not change (NaN makes its group NaN)
    other = kv.PagedCache(_shape(hkv, d, 16), 320, elem_bytes=0.5, fill=0)
    k, v = torch.randn(2, t, hkv, d, device="cuda")
    kv.kv_op_cache_write(other, 0, k, v, slots)
    a, b = torch.empty_like(k), torch.empty_like(v)
    kv.kv_op_cache_read(other, 0, slots, a, b)
    for x, y in ((k, a), (v, b)):
        pick = torch.randint(0, t, (40,))
        for i in pick.tolist():
            assert np.array_equal(P.stored(x[i, i % hkv].cpu().numpy()), _np(y[i, i % hkv]))
        # a value is off by at most half the widest gap between codes (2 of 6) of its group's largest, the scale's step (1/8) above it
        top = x.unflatten(-1, (-1, 16)).abs().amax(-1, keepdim=True)
        assert ((x - y).unflatten(-1, (-1, 16)).abs() <= top * (1.125 / 6) + 2.0 ** -20).all()


@pytest.mark.parametrize("power", [-110, -3, 0, 100])
def test_values_next_to_the_borders_of_codes(kv, torch, power):
    """fp32 rows of values on a border between two codes, and a few units in the last place to either side of it, for scales of every
    significand: the code is the definition's."""
    rng = np.random.default_rng(200 + power)
    t, d, borders = 150, 64, np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    scales = S.e4m3_values()[rng.integers(60, 127, (t, d // 16))]
    scales[:, 0] = 448.0                                              # the row's largest value is 6 * 448 * 2^power
    x = np.float32(np.repeat(scales, 16, 1) * borders[rng.integers(0, 7, (t, d))])
    steps = rng.choice([0, 0, 1, 2, 3, 7, 20, 60], (t, d)) * rng.choice([-1, 1], (t, d))
    x = (x.view(np.int32) + steps.astype(np.int32)).view(np.float32)
    x[:, ::16] = np.float32(6 * scales)                               # sets the group's scale
    x = np.ldexp(x * rng.choice([-1, 1], (t, d)).astype(np.float32), power).astype(np.float32)
    cache = kv.PagedCache(_shape(1, d, 16), 10, elem_bytes=0.5, fill=0)
    rows, slots = torch.from_numpy(x[:, None]).cuda(), torch.arange(t, device="cuda")
    kv.kv_op_cache_write(cache, 0, rows, rows, slots)
    back, other = torch.empty_like(rows), torch.empty_like(rows)
    kv.kv_op_cache_read(cache, 0, slots, back, other)
    for i in range(t):
        assert np.array_equal(P.stored(x[i]), _np(back)[i, 0]), i
    assert torch.equal(back, other)


# ------------------------------------------------------------------ appending
APPEND = [  # tokens, q heads, kv heads, dim, rotary, layout, block, type
    (1, 8, 2, 128, 128, "half", 16, "bfloat16"), (1, 64, 8, 128, 128, "half", 16, "bfloat16"),
    (7, 4, 1, 64, 64, "half", 8, "float32"), (33, 6, 3, 64, 64, "interleaved", 7, "bfloat16"),
    (20, 0, 8, 128, 128, "half", 16, "bfloat16"), (20, 5, 5, 128, 64, "half", 24, "float32"),
    (9, 3, 3, 128, 106, "half", 16, "bfloat16"), (9, 3, 3, 128, 106, "interleaved", 16, "float32"),
    (11, 2, 1, 64, 6, "half", 1, "float32"), (5, 2, 2, 64, 62, "half", 16, "bfloat16"), (5, 40, 2, 128, 96, "half", 32, "bfloat16"),
    (700, 4, 1, 64, 64, "half", 16, "bfloat16"), (900, 3, 2, 128, 128, "half", 16, "float32"), (1300, 0, 2, 128, 128, "interleaved", 16, "bfloat16"),
    (2500, 16, 8, 64, 48, "half", 32, "bfloat16"),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("in_place", [False, True])
def test_append_is_rope_then_write(kv, torch, case, elem, in_place):
    t, hq, hkv, d, rotary, layout, block, dtype = case
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(t)
    rope = kv.Rope(rotary, layout=layout, base=1e6, scaling="parts", factor=8.0, original_ctx=4096, gain=1.2 if t % 2 else 1.0)
    nb = -(-t // block) + 2
    a, b = (kv.PagedCache(_shape(hkv, d, block, 2), nb, elem_bytes=elem, layout="block_major" if t % 3 == 0 else "layer_major") for _ in range(2))
    for c in (a, b):
        c.data.view(torch.uint8).fill_(0x5A)
    qkv = torch.randn(t, hq + 2 * hkv + 1, d, generator=gen, device="cuda") * torch.exp2(
        torch.randint(-9, 9, (t, hq + 2 * hkv + 1, 1), generator=gen, device="cuda").float())
    qkv = qkv.to(dtype)
    qkv[0, hq, 3] = math.inf                                             # a key that is not finite
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:hq + 2 * hkv]
    pos = torch.randint(0, 70000, (t,), generator=gen, device="cuda").to(torch.int32)
    special = torch.tensor([0, 2 ** 31 - 1, -5, -2 ** 31][:t], dtype=torch.int32, device="cuda")
    pos[t - len(special):] = special
    slots = torch.randperm(nb * block, generator=gen, device="cuda")[:t]
    if t > 4:
        slots[1], slots[3] = -1, nb * block
    turned, q_want = torch.empty(t, hkv, d, dtype=dtype, device="cuda"), torch.empty(t, hq, d, dtype=dtype, device="cuda")
    kv.kv_op_rope(rope, k, pos, turned)
    if hq:
        kv.kv_op_rope(rope, q, pos, q_want)
    kv.kv_op_cache_write(a, 1, turned, v, slots)
    before = qkv.clone()
    guard = torch.full((t, hq + 2, d), 7.0, dtype=dtype, device="cuda")
    q_out = q if in_place else guard[:, 1:1 + hq]
    if hq:
        kv.kv_op_cache_append(rope, b, 1, k, v, pos, slots, q=q, q_out=q_out)
    else:
        kv.kv_op_cache_append(rope, b, 1, k, v, pos, slots)
    assert torch.equal(a.data, b.data)
    same = lambda x, y: torch.equal(x.view(torch.uint8), y.contiguous().view(torch.uint8))
    if hq:
        assert same(q_want, q_out)
    assert same(before[:, hq:], qkv[:, hq:]) and (in_place or same(before, qkv))
    assert (guard[:, 0] == 7).all() and (guard[:, hq + 1] == 7).all()


def test_append_against_the_oracle(kv, torch):
    """Turned keys in e2m1 pages: of the values that the oracle's keys, moved by the rotation's error bound either way, may be stored as."""
    t, hq, hkv, d, block = 50, 4, 2, 64, 16
    gen = torch.Generator(device="cuda").manual_seed(1)
    rope = kv.Rope(d, base=1e4)
    cache = kv.PagedCache(_shape(hkv, d, block), 5, elem_bytes=0.5, fill=0)
    q, k, v = (torch.randn(t, h, d, generator=gen, device="cuda") for h in (hq, hkv, hkv))
    pos, slots = torch.arange(t, device="cuda", dtype=torch.int32) + 1000, torch.arange(t, device="cuda") + 13
    q_out = torch.empty_like(q)
    kv.kv_op_cache_append(rope, cache, 0, k, v, pos, slots, q=q, q_out=q_out)
    for x, got in ((q, q_out),):
        want = S.rope(_np(x), pos.cpu().numpy(), rope.frequencies(), "half")
        a = np.abs(_np(x))
        other = np.concatenate([a[..., d // 2:], a[..., :d // 2]], -1)
        assert (np.abs(_np(got) - want) <= (a + other) * (8e-7 + 6 * 2.0 ** -24) + 2.0 ** -24 * np.abs(want)).all()
    ks, vs = torch.empty_like(k), torch.empty_like(v)
    kv.kv_op_cache_read(cache, 0, slots, ks, vs)
    turned = S.rope(_np(k), pos.cpu().numpy(), rope.frequencies(), "half")
    differ = 0
    for i in range(t):
        for h in range(hkv):
            assert np.array_equal(_np(vs)[i, h], P.stored(_np(v)[i, h]))
            differ += int((P.stored(turned[i, h]) != _np(ks)[i, h]).sum())
    # a key changes its code if it lies within 2e-6 of itself of a border: one in 10^5 or fewer, here of 6,400 (and a group its scale
    # likewise: 400 of them)
    assert differ <= 16


# ------------------------------------------------------------------ attention
CASES = sorted({(tuple(c[0]), *c[1:5], c[6]) for c in ATTEND}, key=str)


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}x{c[2]}-{c[3]}-{c[4]}-{c[5]}")
def test_attention(kv, torch, case):
    lens, hkv, group, d, block, dtype = case
    b = Batch(kv, torch, lens, hkv, group, d, block, 0.5, getattr(torch, dtype))
    b.run(kv)
    b.check(torch)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_attention_equal_weights_that_round_alike(kv, torch, d, dtype):
    """All keys of a request are one key, so all its weights are one number, and its rounding does not average out: 2^-11 of the result in
    bf16 calls (one fp16 part), 2^-22 in fp32 calls.  lse takes the weights whole.  Counted with it: the maximum's and the exponential's
    rounding (2^-13 of the largest score, 2^-14 as in Batch.check) touch all weights alike here and cancel but for 2^-22, a rounding of
    each fp32 sum (2^-23 a tile), and the result's own rounding."""
    lens = [1, 2, 3, 15, 16, 17, 40, 63, 200, 511] * 3
    b = Batch(kv, torch, lens, 2, 4, d, 16, 0.5, getattr(torch, dtype))
    table = b.table.cpu().numpy()
    for r, n in enumerate(lens):
        pos = np.arange(n)
        slots = torch.from_numpy(table[r, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
        keys = torch.from_numpy(np.repeat(b.k[r][:1], n, 0).astype(np.float32)).cuda()
        rows = torch.from_numpy(b.v[r][:n].astype(np.float32)).cuda()
        kv.kv_op_cache_write(b.cache, b.layer, keys, rows, slots)
        kv.kv_op_cache_read(b.cache, b.layer, slots, keys, rows)
        b.k[r], b.v[r] = _np(keys), _np(rows)
    b.run(kv)
    out, half = _np(b.out), _half_step(torch, b.q.dtype)
    weight = 2.0 ** -11 if dtype == "bfloat16" else 2.0 ** -22
    for r, n in enumerate(lens):
        o, ls, size, most = S.attend(_np(b.q)[r], b.k[r][:n], b.v[r][:n], d ** -0.5)
        share = weight * 1.01 + (n / 16 + 64) * 2.0 ** -22
        assert (np.abs(out[r] - o) <= size * share + half * np.abs(o) * 1.01).all(), (r, n)
    b.check(torch)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("block", [1, 3, 8, 16, 17, 48, 64])
def test_attention_pages_of_every_size(kv, torch, d, block):
    b = Batch(kv, torch, LENGTHS + [700], 3, 4, d, block, 0.5, torch.float32, layout="block_major", layers=2)
    b.run(kv)
    b.check(torch)


@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("d,block", [(128, 16), (64, 7)])
def test_attention_of_few_whole_contexts(kv, torch, elem, dtype, d, block):
    """Heads enough for an SM each and contexts short enough to stay whole, of every length around the eight warps' rows; and one more
    than that, which is split."""
    lens = [1024, 0, 1, 127, 128, 129, 255, 256, 257, 512, 900, 1023, 16]
    for longest in (1024, 1025):
        b = Batch(kv, torch, [longest] + lens, 8, 3, d, block, elem, getattr(torch, dtype))
        b.run(kv)
        b.check(torch)
        first = b.out.clone()
        b.run(kv)
        assert torch.equal(first, b.out)


@pytest.mark.parametrize("many", [False, True])
def test_attention_rows_of_very_different_sizes(kv, torch, many):
    """Scales of K and V rows spread over 2^-12 .. 2^4, and values 2^20 times larger where the scores are lowest: a weight near zero on a
    huge row must not cost the others their bits."""
    lens = [900, 33] + ([50] * 120 if many else [])
    b = Batch(kv, torch, lens, 8, 2, 128, 16, 0.5, torch.float32, sizes=(-12, 4), q_size=0.2)
    b.run(kv)
    b.check(torch)
    s = np.einsum("hd,nd->hn", _np(b.q)[0][:2], b.k[0][:, 0])
    rows = torch.from_numpy(b.v[0].astype(np.float32)).cuda()
    rows[np.argsort(s.max(0))[:40]] *= 2.0 ** 20
    pos, table = np.arange(lens[0]), b.table.cpu().numpy()
    slots = torch.from_numpy(table[0, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
    keys = torch.from_numpy(b.k[0].astype(np.float32)).cuda()
    kv.kv_op_cache_write(b.cache, 0, keys, rows, slots)
    back = torch.empty_like(rows)
    kv.kv_op_cache_read(b.cache, 0, slots, keys, back)
    b.k[0], b.v[0] = _np(keys), _np(back)
    b.run(kv)
    b.check(torch)


def test_attention_extreme_scores_and_scale(kv, torch):
    b = Batch(kv, torch, [700, 20], 2, 4, 128, 16, 0.5, torch.float32, q_size=4.0)
    b.run(kv, softmax_scale=0.5)
    b.check(torch, scale=0.5)
    b.q.zero_()
    b.run(kv)
    b.check(torch)


@pytest.mark.parametrize("many", [False, True])
def test_attention_ids_outside_the_pool_and_lengths_outside_the_range(kv, torch, many):
    lens = [100, 90, 600, 64] + ([33] * 90 if many else [])
    b = Batch(kv, torch, lens, 8, 2, 64, 16, 0.5, torch.float32)
    b.table[1, 3], b.table[2, 20] = b.cache.num_blocks, -1
    b.lens_dev[0], b.lens_dev[3] = 10 ** 6, -4           # clamped to max_ctx: a table of -1 behind its blocks; to 0
    b.run(kv)
    assert torch.isnan(b.out[:3]).all() and torch.isnan(b.lse[:3]).all()
    assert (b.out[3] == 0).all() and (b.lse[3] == -math.inf).all()
    b.check(torch, only=range(4, len(lens)))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("many", [False, True])
def test_attention_infinite_and_nan_inputs(kv, torch, d, many):
    """A key that was not finite makes NaN of the heads of its group, a value of the 16 dims of its scale, a query of its head, and of
    nothing else; rows behind a context (NaN everywhere in these pages) of nothing."""
    lens = [200, 70, 600, 40] + ([33] * 90 if many else [])
    b = Batch(kv, torch, lens, 4, 2, d, 16, 0.5, torch.float32)
    b.run(kv)
    clean, clean_lse = b.out.clone(), b.lse.clone()

    def put(r, at, h, key=None, value=None):
        slot = (b.table[r, at // 16].long() * 16 + at % 16).view(1)
        k = torch.from_numpy(b.k[r][at:at + 1].astype(np.float32)).cuda()
        v = torch.from_numpy(b.v[r][at:at + 1].astype(np.float32)).cuda()
        if key is not None:
            k[0, h, 5] = key
        if value is not None:
            v[0, h, 37] = value
        kv.kv_op_cache_write(b.cache, 0, k, v, slot)
    put(0, 199, 1, key=math.inf)
    put(1, 3, 2, value=math.nan)
    put(2, 300, 0, value=-math.inf)
    b.q[3, 5, 7] = math.nan
    b.run(kv)
    want, want_lse = clean.clone(), clean_lse.clone()
    want[0, 2:4], want_lse[0, 2:4] = math.nan, math.nan
    want[1, 4:6, 32:48] = math.nan
    want[2, 0:2, 32:48] = math.nan
    want[3, 5], want_lse[3, 5] = math.nan, math.nan
    assert torch.equal(torch.isnan(b.out), torch.isnan(want)) and torch.equal(torch.isnan(b.lse), torch.isnan(want_lse))
    # a row that holds a NaN leaves it out of its scales, so what it stores elsewhere keeps its bits where no other maximum fell away
    keep = [r for r in range(len(lens)) if r not in (0, 1, 2)]
    assert torch.equal(b.out[keep].nan_to_num(7), want[keep].nan_to_num(7))


def test_attention_far_offsets(kv, torch):
    """Pages whose byte offsets pass 32 bits."""
    page = kv.kv_cache_page_bytes(16, 8, 128, 0.5)
    nb = (1 << 32) // page + 40
    cache = kv.PagedCache(_shape(8, 128, 16), nb, elem_bytes=0.5)
    n = 600
    rows = torch.randn(2, n, 8, 128, device="cuda")
    table = (nb - 1 - torch.arange(38, device="cuda", dtype=torch.int32)).view(1, -1)
    pos = torch.arange(n, device="cuda")
    slots = table[0].long()[pos // 16] * 16 + pos % 16
    rope = kv.Rope(128)
    kv.kv_op_cache_append(rope, cache, 0, rows[0], rows[1], torch.zeros(n, dtype=torch.int32, device="cuda"), slots)      # not turned
    back = torch.empty_like(rows)
    kv.kv_op_cache_read(cache, 0, slots, back[0], back[1])
    assert float((back - rows).abs().max()) < 1.0
    q = torch.randn(1, 16, 128, device="cuda") * 0.3
    out, lse = torch.empty_like(q), torch.empty(1, 16, device="cuda")
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(1, 16, cache, n), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, table, torch.tensor([n], dtype=torch.int32, device="cuda"), n, out, scratch, lse=lse)
    o, ls, size, most = S.attend(_np(q)[0], _np(back[0]), _np(back[1]), 128 ** -0.5)
    share = most * 2.0 ** -13 + 2.0 ** -14 + 102 * 2.0 ** -22
    assert (np.abs(_np(out)[0] - o) <= size * share).all()


def test_attention_same_bits_every_time_in_place_and_strided(kv, torch):
    b = Batch(kv, torch, [1200, 40, 0, 513], 2, 4, 128, 16, 0.5, torch.bfloat16)
    b.run(kv)
    first = (b.out.clone(), b.lse.clone())
    for _ in range(5):
        b.scratch.fill_(0xFF)
        b.run(kv)
        assert torch.equal(b.out, first[0]) and torch.equal(b.lse, first[1])
    wide = torch.full((4, 20, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 4:12] = b.q
    kv.kv_op_paged_attention_batched(wide[:, 4:12], b.cache, 0, b.table, b.lens_dev, b.ctx, wide[:, 4:12], b.scratch)
    assert torch.equal(wide[:, 4:12], first[0]) and (wide[:, :4] == 7).all() and (wide[:, 12:] == 7).all()


# ------------------------------------------------------------------ pages on the wire, graphs, streams
@pytest.mark.parametrize("case", [(8, 128, 16), (3, 64, 7), (8, 128, 64), (2, 64, 16), (1, 64, 4)], ids=str)
def test_e2m1_pages_travel_whole(kv, torch, case):
    hkv, d, block = case
    shape = _shape(hkv, d, block, layers=2)
    for layout in ("layer_major", "block_major"):
        src, dst = (kv.PagedCache(shape, 13, layout=layout, elem_bytes=0.5) for _ in range(2))
        src.data.copy_(torch.randint(0, 256, src.data.shape, device="cuda", dtype=torch.uint8))
        dst.data.fill_(0xA5)
        ids, to = [7, 0, 12, 3, 5], [1, 11, 4, 2, 9]
        wire = torch.full((5 * 4 * src.page_bytes + 64,), 0x3C, dtype=torch.uint8, device="cuda")
        kv.kv_pack_blocks_batched(src, [0, 3, 5], ids, [wire, wire[3 * 4 * src.page_bytes:]])
        kv.kv_unpack_blocks_batched(dst, [0, 3, 5], to, [wire, wire[3 * 4 * src.page_bytes:]])
        kv.kv_check_copy_status()
        a, b = _pages_numpy(src), _pages_numpy(dst)
        assert np.array_equal(a[:, :, ids], b[:, :, to]) and (wire[-64:] == 0x3C).all()
        assert (b[:, :, np.setdiff1d(np.arange(13), to)] == 0xA5).all()


def test_e2m1_suffix_streams_to_the_target(kv, torch):
    """Suffix streaming of a 4-bit cache, its tokens appended one by one: the target's pages equal the source's."""
    from paper_2608_16477_b200 import streaming
    shape = _shape(2, 64, 16, layers=2)
    src, tgt = (kv.PagedCache(shape, 20, elem_bytes=0.5, fill=0) for _ in range(2))
    perm, fresh = np.random.default_rng(3).permutation(20), np.random.default_rng(4).permutation(20)
    k, n = 32, 32 + 53
    table = perm[:-(-n // 16)]
    rope = kv.Rope(64)
    rx = streaming.SuffixReceiver(tgt, request_id=1, expected_epoch=2, k_split=k, max_suffix_blocks=6, fresh_block_ids=fresh[2:10])
    tx = streaming.SuffixStreamer(src, table, k, request_id=1, epoch=2, transport=streaming.LoopbackTransport(rx))
    for pos in range(n):
        rows = torch.randn(2, 1, 2, 64, device="cuda")
        slots = torch.tensor([int(table[pos // 16]) * 16 + pos % 16], device="cuda")
        at = torch.tensor([pos], dtype=torch.int32, device="cuda")
        for layer in range(2):
            kv.kv_op_cache_append(rope, src, layer, rows[0], rows[1] + layer, at, slots)
        if pos >= k:
            tx.on_token(pos)
            if pos % 20 == 0:
                tx.pump(max_blocks=1)
    tx.final_sync(n)
    merged = rx.assemble(fresh[:2], n, epoch=2)
    torch.cuda.synchronize()
    a, b = _pages_numpy(src), _pages_numpy(tgt)
    assert np.array_equal(a[:, :, table[2:]], b[:, :, merged[2:]]) and a[:, :, table[2:]].any()


def test_captured_append_and_attention_replay_with_new_lists(kv, torch):
    """A decode step's append and attention in one graph, replayed token after token with new positions, slots and lengths."""
    r, hq, hkv, d, block, steps = 3, 8, 2, 64, 16, 40
    gen = torch.Generator(device="cuda").manual_seed(5)
    rope = kv.Rope(d, base=1e4)
    caches = [kv.PagedCache(_shape(hkv, d, block), 12, elem_bytes=0.5, fill=0) for _ in range(2)]
    table = torch.randperm(12, generator=gen, device="cuda").to(torch.int32).view(3, 4)
    qkv = torch.zeros(r, hq + 2 * hkv, d, dtype=torch.bfloat16, device="cuda")
    pos, slots = torch.zeros(r, dtype=torch.int32, device="cuda"), torch.zeros(r, dtype=torch.int64, device="cuda")
    lens = torch.zeros(r, dtype=torch.int32, device="cuda")
    q, out = torch.empty(r, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(r, hq, d, dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(r, hq, caches[0], 64), dtype=torch.uint8, device="cuda")

    def step(cache):
        kv.kv_op_cache_append(rope, cache, 0, qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], pos, slots, q=qkv[:, :hq], q_out=q)
        kv.kv_op_paged_attention_batched(q, cache, 0, table, lens, 64, out, scratch)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(caches[1])
    torch.cuda.current_stream().wait_stream(side)
    caches[1].data.zero_()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(caches[0])
    caches[0].data.zero_()
    start = torch.tensor([0, 5, 20], dtype=torch.int32, device="cuda")
    for i in range(steps):
        qkv.copy_(torch.randn(qkv.shape, generator=gen, device="cuda"))
        pos.copy_(start + i)
        slots.copy_(table.gather(1, (pos // block).long()[:, None])[:, 0].long() * block + pos % block)
        lens.copy_(pos + 1)
        graph.replay()
        got = out.clone()
        step(caches[1])
        assert torch.equal(got.view(torch.int16), out.view(torch.int16))
    assert torch.equal(caches[0].data, caches[1].data)
