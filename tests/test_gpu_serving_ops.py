"""The batch-serving operators on the GPU against the fp64 oracle (oracle/serving_oracle.py).

Tolerances.  A rounding to type t is off by at most finfo(t).eps / 2 of the value.
  rotary positions: the angle is off by at most 2^-24 turn in its reduction and 2^-24 of itself (at most half a turn) in
    its rounding to fp32, so by 2 pi 2^-23 < 8e-7; sine and cosine by 2 ulp; the products and the sum by 3 roundings:
    |error| <= gain (|a| + |b|) (8e-7 + 6 * 2^-24) and the rounding of the result.
  pages: exact.
  attention: A = the largest scale * sum |q_i k_i| of a request.  q is held in two bf16 (2^-16 of each term; fp16: less),
    the products are summed in fp32 (d + 8 roundings of 2^-24 at the worst, all of them towards A), so a score is off by at
    most A (2^-16 + 136 * 2^-24) < A 2^-15 and a weight and the sum of weights by that share each; weights are held in two
    bf16 (2^-16) and ex2 is off by 2^-22 and the rounding of its argument (2^-24 of at most 1.5 (A + |max|), inside the A
    term); partial sums are added in at most n / 16 + 64 fp32 steps.  With B = sum p |v| / sum p:
    |error| <= B (A 2^-13 + 2^-14 + (n / 16 + 64) 2^-22) and the rounding of the result; lse: the same without B.
"""
import math

import numpy as np
import pytest

import synth
from oracle import serving_oracle as S

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


def _half_step(torch, dtype):
    return torch.finfo(dtype).eps / 2


def _np(t):
    return t.double().cpu().numpy()


def _shape(kv_heads, dim, block, layers=1):
    return synth.ModelShape("serve", n_layers=layers, hidden=64, n_q_heads=kv_heads, n_kv_heads=kv_heads, head_dim=dim,
                            ffn=64, vocab=16, block_size=block)


# ------------------------------------------------------------------ rotary positions
ROPE = [  # tokens, heads, head_dim, rotary, layout, scaling, dtype, arrangement
    (1, 1, 64, 64, "half", dict(), "bfloat16", "plain"),
    (3, 5, 128, 128, "half", dict(scaling="ntk", factor=8.0), "bfloat16", "plain"),
    (1, 72, 128, 128, "half", dict(), "float32", "qkv"),
    (37, 9, 128, 64, "interleaved", dict(scaling="linear", factor=8.0), "bfloat16", "qkv"),
    (130, 3, 128, 96, "half", dict(scaling="parts", factor=8.0, original_ctx=4096, gain=1.2), "bfloat16", "heads"),
    (18, 4, 64, 16, "interleaved", dict(), "float32", "heads"),
    (5, 3, 64, 50, "half", dict(), "bfloat16", "plain"),             # pairs that fill no vector
    (5, 3, 80, 50, "interleaved", dict(), "float32", "plain"),
    (7, 2, 64, 64, "half", dict(), "bfloat16", "odd"),               # rows that start on no vector
    (7, 2, 64, 32, "interleaved", dict(), "float32", "odd"),
    (9, 2, 65, 64, "half", dict(), "float32", "plain"),
    (700, 2, 256, 256, "half", dict(), "bfloat16", "plain"),
    (2500, 3, 64, 64, "interleaved", dict(), "bfloat16", "plain"),   # several tokens to a CTA, the last one short
    (4, 40, 64, 2, "half", dict(), "float32", "plain"),
    (19, 21, 128, 102, "half", dict(), "bfloat16", "qkv"),           # halves that start on different places of a vector
    (19, 9, 128, 102, "interleaved", dict(), "bfloat16", "qkv"),     # ... and pairs that end inside one
    (700, 3, 1024, 250, "half", dict(), "float32", "heads"),
    (6, 5, 72, 70, "interleaved", dict(), "bfloat16", "plain"),
    (6, 5, 72, 72, "interleaved", dict(), "float32", "plain"),
    (3, 19, 1024, 6, "half", dict(), "bfloat16", "plain"),
    (2, 3, 68, 66, "half", dict(), "float32", "heads"),
]


def _rope_rows(torch, t, h, d, dtype, arrangement, gen):
    if arrangement == "qkv":
        return torch.randn(t, h + 7, d, generator=gen, device="cuda").to(dtype)[:, 3:3 + h]
    if arrangement == "heads":
        return torch.randn(h, t, d, generator=gen, device="cuda").to(dtype).transpose(0, 1)
    if arrangement == "odd":
        return torch.randn(t, h, d + 1, generator=gen, device="cuda").to(dtype)[..., 1:]
    return torch.randn(t, h, d, generator=gen, device="cuda").to(dtype)


@pytest.mark.parametrize("case", ROPE, ids=lambda c: f"{c[0]}x{c[1]}x{c[2]}-{c[3]}-{c[4]}-{c[6]}-{c[7]}")
@pytest.mark.parametrize("backward", [False, True])
@pytest.mark.parametrize("in_place", [False, True])
def test_rope(kv, torch, case, backward, in_place):
    t, h, d, rotary, layout, kw, dtype, arrangement = case
    dtype = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = _rope_rows(torch, t, h, d, dtype, arrangement, gen)
    pos = torch.randint(0, 70000, (t,), generator=gen, device="cuda").to(torch.int32)
    special = torch.tensor([0, 2**31 - 1, -5, -2**31, 1][:t], dtype=torch.int32, device="cuda")
    pos[:len(special)] = special
    rope = kv.Rope(rotary, layout=layout, base=1e6, **kw)
    gain = kw.get("gain", 1.0)
    xs = _np(x)
    want = S.rope(xs, pos.cpu().numpy(), rope.frequencies(), layout, gain, backward)
    guard = torch.full((t, h, d + 16), 7.0, dtype=dtype, device="cuda")
    out = x if in_place else guard[..., 8:8 + d]
    kv.kv_op_rope(rope, x, pos, out, backward=backward)
    got = _np(out)
    assert np.array_equal(got[..., rotary:], xs[..., rotary:])
    half = rotary // 2
    a = np.abs(xs[..., :rotary])
    other = np.concatenate([a[..., half:], a[..., :half]], -1) if layout == "half" else a.reshape(t, h, half, 2)[..., ::-1].reshape(a.shape)
    # the oracle's own fp64 angle is off by 2^-53 of up to 2^31 radians: 3e-7 more
    tol = gain * (a + other) * (8e-7 + 3e-7 + 6 * 2.0 ** -24) + _half_step(torch, dtype) * np.abs(want[..., :rotary])
    assert (np.abs(got - want)[..., :rotary] <= tol * (1 + 2.0 ** -10)).all()
    if not in_place:
        assert (guard[..., :8] == 7).all() and (guard[..., 8 + d:] == 7).all()


def test_rope_backward_is_the_gradient(kv, torch):
    """<R x, y> = <x, R^T y>, and R^T y against differences of the loss <R x, y> in single coordinates."""
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, y = torch.randn(2, 11, 3, 64, generator=gen, device="cuda")
    pos = torch.arange(11, device="cuda", dtype=torch.int32) * 321
    for layout in ("half", "interleaved"):
        rope = kv.Rope(48, layout=layout, scaling="parts", factor=4.0, original_ctx=1000, gain=1.1)
        f, g = torch.empty_like(x), torch.empty_like(x)
        kv.kv_op_rope(rope, x, pos, f)
        kv.kv_op_rope(rope, y, pos, g, backward=True)
        a, b = (f.double() * y.double()), (x.double() * g.double())
        assert abs(float(a.sum() - b.sum())) <= 2e-6 * float(a.abs().sum() + b.abs().sum())
        for t, h, i in ((0, 0, 0), (5, 1, 23), (10, 2, 40), (7, 0, 63)):
            e = torch.zeros_like(x)
            e[t, h, i] = 1.0
            up, down = torch.empty_like(x), torch.empty_like(x)
            kv.kv_op_rope(rope, x + e, pos, up)
            kv.kv_op_rope(rope, x - e, pos, down)
            diff = float(((up.double() - down.double()) * y.double()).sum() / 2)
            # both sides carry fp32 roundings of values of size |x| + 1 over the two coordinates of the pair
            assert abs(diff - float(g[t, h, i])) <= 1e-5 * (2 + float(x[t, h].abs().max())) * (1 + float(y[t, h].abs().max()))


def test_rope_of_a_broadcast_row_and_of_no_tokens(kv, torch):
    rope = kv.Rope(64)
    x = torch.randn(1, 1, 64, device="cuda").expand(6, 3, 64)
    pos = torch.arange(6, device="cuda", dtype=torch.int32)
    out, want = torch.empty(6, 3, 64, device="cuda"), torch.empty(6, 3, 64, device="cuda")
    kv.kv_op_rope(rope, x, pos, out)
    kv.kv_op_rope(rope, x.contiguous(), pos, want)
    assert torch.equal(out, want)
    kv.kv_op_rope(rope, x[:0], pos[:0], out[:0])


# ------------------------------------------------------------------ rows into pages and back
def _pages_numpy(cache):
    """raw bytes [L, 2, blocks, page bytes]."""
    d = cache.data.view(-1).view(dtype=cache.data.dtype).reshape(cache.data.shape)
    if cache.layout == "block_major":
        d = d.permute(1, 2, 0, 3)
    return d.contiguous().cpu().numpy().view(np.uint8).reshape(cache.n_layers, 2, cache.num_blocks, cache.page_bytes)


def _expected_row(x, elem, torch):
    """(bytes of the row, scale byte or None)."""
    if elem == 2:
        return torch.from_numpy(np.ascontiguousarray(x)).to(torch.bfloat16).view(torch.uint8).numpy(), None
    codes, byte = S.quantise_row(x)
    return codes, byte


def _special_rows(d):
    """Rows at the borders of the format."""
    rng = np.random.default_rng(7)
    base = rng.standard_normal(d).astype(np.float32)
    rows = [base * 0, base, -base]
    for top in (448.0, 448.5, 447.9, 224.0, 224.1, 2.0 ** -100, 3.0e38, 2.0 ** -126, 1e-40, 3.3895e38):
        r = base / 8
        r = np.where(np.abs(r) >= 1, 0.5, r).astype(np.float32) * np.float32(min(top, 1e30))
        r[3] = top
        rows.append(r)
    r = base.copy(); r[0] = np.inf; r[5] = -np.inf; r[7] = np.nan
    rows.append(r)
    rows.append(np.full(d, np.nan, np.float32))
    rows.append(np.full(d, -np.inf, np.float32))
    ties = (np.arange(d) + 16.5).astype(np.float32) * 8      # half-way values between codes
    ties[-1] = 448 * 4
    rows.append(ties)
    rows.append(np.float32(2.0 ** -9) * (np.arange(d) + 0.5).astype(np.float32))     # subnormal codes
    r = np.zeros(d, np.float32); r[::2] = -0.0; r[1] = 448
    rows.append(r)
    return np.stack(rows).astype(np.float32)


WRITE = [  # tokens, kv_heads, dim, block, layers, layout
    (1, 1, 64, 16, 1, "layer_major"), (5, 8, 128, 16, 2, "layer_major"), (67, 3, 64, 7, 2, "block_major"),
    (333, 2, 128, 32, 1, "layer_major"), (40, 8, 64, 1, 3, "block_major"), (129, 5, 128, 24, 1, "layer_major"),
]


@pytest.mark.parametrize("case", WRITE, ids=lambda c: "-".join(map(str, c)))
@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_write_then_read(kv, torch, case, elem, dtype):
    t, hkv, d, block, layers, layout = case
    dtype = getattr(torch, dtype)
    rng = np.random.default_rng(t)
    nb = -(-t // block) + 3
    cache = kv.PagedCache(_shape(hkv, d, block, layers), nb, layout=layout, elem_bytes=elem)
    cache.data.view(torch.uint8).fill_(0x5A)
    before = _pages_numpy(cache).copy()
    x = rng.standard_normal((2, t, hkv, d)).astype(np.float32) * 2.0 ** rng.integers(-30, 30, (2, t, hkv, 1)).astype(np.float32)
    special = _special_rows(d)
    for i in range(min(t * hkv, len(special))):
        x[i % 2, i // hkv, i % hkv] = special[i]
    both = torch.from_numpy(x).cuda().to(dtype)
    order = rng.permutation(nb * block)[:t].astype(np.int64)
    slots = torch.from_numpy(order.copy()).cuda()
    if t > 4:
        slots[2], slots[4] = -1, nb * block          # padding and a slot behind the pool: left out
    layer = layers - 1
    # K out of a wide buffer, V head-major
    wide = torch.zeros(t, 3 * hkv, d, dtype=dtype, device="cuda")
    wide[:, hkv:2 * hkv] = both[0]
    k, v = wide[:, hkv:2 * hkv], both[1].transpose(0, 1).contiguous().transpose(0, 1)
    kv.kv_op_cache_write(cache, layer, k, v, slots)
    after = _pages_numpy(cache)
    want = before.copy()
    xs = both.float().cpu().numpy()
    values = block * hkv * d * elem
    table = S.e4m3_values()
    decoded = np.zeros((2, t, hkv, d))
    for i, s in enumerate(slots.cpu().tolist()):
        for h in range(hkv):
            for c in range(2):
                raw, byte = _expected_row(xs[c, i, h], elem, torch)
                decoded[c, i, h] = table[raw] * 2.0 ** (byte - 127.0) if elem == 1 else \
                    torch.from_numpy(raw.copy()).view(torch.bfloat16).double().numpy()
                if not 0 <= s < nb * block:
                    continue
                b, o = divmod(s, block)
                at = (o * hkv + h) * d * elem
                want[layer, c, b, at:at + d * elem] = raw
                if elem == 1:
                    want[layer, c, b, values + h * block + o] = byte
    if elem == 2:        # NaN keeps no particular payload
        a, w = after[..., :values].view(np.uint16), want[..., :values].view(np.uint16)
        nan = lambda u: (u & 0x7FFF) > 0x7F80
        assert ((a == w) | (nan(a) & nan(w))).all()
    else:
        assert np.array_equal(after, want)
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


def test_rows_of_no_tokens(kv, torch):
    cache = kv.PagedCache(_shape(2, 64, 16), 2, elem_bytes=1, fill=9)
    rows, slots = torch.empty(0, 2, 64, device="cuda"), torch.empty(0, dtype=torch.int64, device="cuda")
    kv.kv_op_cache_write(cache, 0, rows, rows, slots)
    kv.kv_op_cache_read(cache, 0, slots, rows, rows)
    assert (cache.data == 9).all()


# ------------------------------------------------------------------ attention
class Batch:
    """Requests over a shuffled pool; pages hold NaN wherever no context reaches."""

    def __init__(self, kv, torch, lens, hkv, group, d, block, elem, dtype, seed=0, layers=1, layout="layer_major",
                 spare=3, sizes=None, q_size=0.3, ctx=None):
        rng = np.random.default_rng(seed)
        self.lens, self.hkv, self.group, self.d = list(lens), hkv, group, d
        need = [-(-n // block) for n in lens]
        self.ctx = ctx or max(max(lens), 1)
        nb = sum(need) + spare
        self.cache = kv.PagedCache(_shape(hkv, d, block, layers), nb, layout=layout, elem_bytes=elem)
        raw = self.cache.data.view(torch.uint8)
        raw.fill_(0xFF)                                # bf16 0xffff and code 0xff are NaN
        self.layer = layers - 1
        cols = max(max(need), -(-self.ctx // block))
        table = np.full((len(lens), cols), -1, dtype=np.int32)
        order = rng.permutation(nb)
        at = 0
        for r, n in enumerate(need):
            table[r, :n] = order[at:at + n]
            at += n
        self.k, self.v = [], []
        for r, n in enumerate(lens):
            x = rng.standard_normal((2, n, hkv, d)).astype(np.float32)
            if sizes is not None:
                x *= 2.0 ** rng.integers(sizes[0], sizes[1], (2, n, hkv, 1)).astype(np.float32)
            rows = torch.from_numpy(x).cuda().to(torch.bfloat16)
            pos = np.arange(n)
            slots = torch.from_numpy((table[r, pos // block].astype(np.int64) * block + pos % block)).cuda()
            kv.kv_op_cache_write(self.cache, self.layer, rows[0], rows[1], slots)
            back = torch.empty(2, n, hkv, d, device="cuda")
            kv.kv_op_cache_read(self.cache, self.layer, slots, back[0], back[1])
            self.k.append(_np(back[0]))
            self.v.append(_np(back[1]))
        self.table = torch.from_numpy(table).cuda()
        self.lens_dev = torch.tensor(lens, dtype=torch.int32, device="cuda")
        self.q = torch.from_numpy(rng.standard_normal((len(lens), hkv * group, d)).astype(np.float32) * q_size).cuda().to(dtype)
        need = kv.kv_paged_attention_batched_scratch_bytes(len(lens), hkv * group, self.cache, self.ctx)
        self.scratch = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")     # NaN: nothing may be read unwritten
        self.out = torch.full_like(self.q, 7.0)
        self.lse = torch.full(self.q.shape[:2], 7.0, device="cuda")

    def run(self, kv, **kw):
        kw = {**dict(lse=self.lse), **kw}
        kv.kv_op_paged_attention_batched(self.q, self.cache, self.layer, self.table, self.lens_dev, self.ctx, self.out,
                                         self.scratch, **kw)

    def check(self, torch, scale=None, lens=None, only=None):
        scale = self.d ** -0.5 if scale is None else scale
        q, out, lse = _np(self.q), _np(self.out), _np(self.lse)
        half = _half_step(torch, self.q.dtype)
        for r, n in enumerate(self.lens if lens is None else lens):
            if only is not None and r not in only:
                continue
            o, ls, size, most = S.attend(q[r], self.k[r][:n], self.v[r][:n], scale)
            steps = (n / 16 + 64) * 2.0 ** -22
            share = most * 2.0 ** -13 + 2.0 ** -14 + steps
            err = np.abs(out[r] - o)
            assert (err <= size * share + half * np.abs(o) * 1.01).all(), (r, n, err.max(), (size * share).min())
            if n == 0:
                assert (lse[r] == -np.inf).all()
            else:
                assert (np.abs(lse[r] - ls) <= share + 2.0 ** -23 * np.abs(ls)).all(), (r, n)


LENGTHS = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 200]
ATTEND = [  # lens, kv_heads, group, dim, block, elem, dtype
    ([1], 1, 1, 64, 16, 2, "float32"),
    ([161], 2, 2, 64, 16, 2, "float32"),
    ([161], 2, 2, 64, 16, 1, "bfloat16"),
    (LENGTHS, 2, 4, 128, 16, 2, "bfloat16"),
    (LENGTHS, 2, 4, 128, 16, 1, "float32"),
    (LENGTHS, 3, 8, 64, 8, 1, "bfloat16"),
    (LENGTHS, 3, 3, 64, 8, 2, "float32"),
    ([300, 0, 511, 512, 5], 2, 12, 128, 7, 1, "float32"),        # two passes over the heads, pages that end inside a stage
    ([300, 0, 511, 512, 5], 2, 12, 64, 7, 2, "float32"),
    ([513], 1, 8, 128, 16, 1, "float32"),                        # split
    ([513, 0, 1], 1, 8, 128, 16, 2, "float32"),
    ([4000], 8, 8, 128, 16, 1, "bfloat16"),
    ([4000], 8, 8, 128, 16, 2, "float32"),
    ([2000, 3, 0, 777, 1024, 64], 8, 8, 128, 16, 1, "float32"),
    ([2000, 3, 0, 777, 1024, 64], 8, 4, 64, 32, 1, "float32"),
    ([2000, 3, 0, 777, 1024, 64], 8, 4, 64, 1, 2, "bfloat16"),
    ([700, 90, 1300], 5, 20, 128, 24, 1, "float32"),
    ([1, 600] + [40, 0, 7] * 40, 8, 2, 64, 16, 1, "float32"),    # a warp per KV head
    ([1, 600] + [40, 0, 7] * 40, 8, 2, 128, 16, 2, "float32"),
    ([5, 30] * 110, 3, 1, 64, 5, 1, "bfloat16"),                 # ... with KV heads that fill no CTA
    ([5, 530] * 110, 3, 1, 64, 5, 2, "float32"),
    ([5, 530] * 110, 3, 9, 64, 5, 1, "float32"),
    ([1500] + [0] * 700, 2, 1, 64, 16, 2, "float32"),            # more requests than a scan's round, nearly all empty
]


@pytest.mark.parametrize("case", ATTEND, ids=lambda c: f"{len(c[0])}x{max(c[0])}-{c[1]}x{c[2]}-{c[3]}-{c[4]}-{c[5]}-{c[6]}")
def test_attention(kv, torch, case):
    lens, hkv, group, d, block, elem, dtype = case
    b = Batch(kv, torch, lens, hkv, group, d, block, elem, getattr(torch, dtype))
    b.run(kv)
    b.check(torch)


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("kw", [0, 1])
def test_attention_rows_of_very_different_sizes(kv, torch, elem, kw):
    """Scales of K and V rows spread over 2^-20 .. 2^20 (V) next to one another: a weight near zero on a huge value row
    must not cost the others their bits."""
    lens = [900, 33] if kw == 0 else [900, 33] + [50] * 120
    b = Batch(kv, torch, lens, 8, 2, 128, 16, elem, torch.float32, sizes=(-12, 4), q_size=0.2)
    b.run(kv)
    b.check(torch)
    # V alone: rebuild request 0's values 2^20 times larger where its scores are lowest
    q = _np(b.q)[0]
    s = np.einsum("hd,nd->hn", q[:2], b.k[0][:, 0])
    low = np.argsort(s.max(0))[:40]
    rows = torch.from_numpy(b.v[0].astype(np.float32)).cuda()
    rows[low] *= 2.0 ** 20
    pos = np.arange(lens[0])
    table = b.table.cpu().numpy()
    slots = torch.from_numpy(table[0, pos // 16].astype(np.int64) * 16 + pos % 16).cuda()
    keys = torch.from_numpy(b.k[0].astype(np.float32)).cuda()
    kv.kv_op_cache_write(b.cache, 0, keys, rows, slots)
    back = torch.empty_like(rows)
    kv.kv_op_cache_read(b.cache, 0, slots, keys, back)
    b.k[0], b.v[0] = _np(keys), _np(back)
    b.run(kv)
    b.check(torch)


@pytest.mark.parametrize("elem", [1, 2])
def test_attention_extreme_scores_and_scale(kv, torch, elem):
    """Peaked softmaxes (scores to 80), all scores equal, and a scale of the caller's."""
    b = Batch(kv, torch, [700, 20], 2, 4, 128, 16, elem, torch.float32, q_size=4.0)
    b.run(kv, softmax_scale=0.5)
    b.check(torch, scale=0.5)
    b.q.zero_()
    b.run(kv)
    b.check(torch)


def test_attention_strided_and_without_lse(kv, torch):
    b = Batch(kv, torch, [70, 0, 640], 2, 4, 64, 16, 1, torch.bfloat16)
    wide = torch.full((3, 20, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 4:12] = b.q
    outs = torch.full((3, 24, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    tab = torch.full((3, b.table.shape[1] + 5), 10**9, dtype=torch.int32, device="cuda")
    tab[:, :b.table.shape[1]] = b.table
    kv.kv_op_paged_attention_batched(wide[:, 4:12], b.cache, 0, tab[:, :b.table.shape[1]], b.lens_dev, b.ctx,
                                     outs[:, 8:16], b.scratch)
    assert (outs[:, :8] == 7).all() and (outs[:, 16:] == 7).all() and (b.lse == 7).all()
    b.run(kv)
    assert torch.equal(outs[:, 8:16], b.out)


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("many", [False, True])
def test_attention_ids_outside_the_pool_and_lengths_outside_the_range(kv, torch, elem, many):
    lens = [100, 90, 600, 64] + ([33] * 90 if many else [])
    b = Batch(kv, torch, lens, 8, 2, 64, 16, elem, torch.float32)
    b.table[1, 3], b.table[2, 20] = b.cache.num_blocks, -1
    b.lens_dev[0], b.lens_dev[3] = 10**6, -4           # clamped to max_ctx: a table of -1 behind its blocks; to 0
    b.run(kv)
    assert torch.isnan(b.out[:3]).all() and torch.isnan(b.lse[:3]).all()
    assert (b.out[3] == 0).all() and (b.lse[3] == -math.inf).all()
    b.check(torch, only=range(4, len(lens)))


def test_attention_shared_pages_and_no_requests(kv, torch):
    """Two requests over the same blocks (a shared prefix), and an empty batch."""
    b = Batch(kv, torch, [300, 300], 2, 2, 64, 16, 1, torch.float32)
    b.table[1] = b.table[0]
    b.k[1], b.v[1] = b.k[0], b.v[0]
    b.run(kv)
    b.check(torch)
    kv.kv_op_paged_attention_batched(b.q[:0], b.cache, 0, b.table[:0], b.lens_dev[:0], b.ctx, b.out[:0], b.scratch)


@pytest.mark.parametrize("elem", [1, 2])
def test_attention_far_offsets(kv, torch, elem):
    """Pages whose byte offsets pass 32 bits."""
    s = _shape(8, 128, 16)
    page = kv.kv_cache_page_bytes(16, 8, 128, elem)
    nb = (1 << 32) // page + 40
    cache = kv.PagedCache(s, nb, elem_bytes=elem)
    n = 600
    rows = torch.randn(2, n, 8, 128, device="cuda")
    table = (nb - 1 - torch.arange(38, device="cuda", dtype=torch.int32)).view(1, -1)
    pos = torch.arange(n, device="cuda")
    slots = table[0].long()[pos // 16] * 16 + pos % 16
    kv.kv_op_cache_write(cache, 0, rows[0], rows[1], slots)
    back = torch.empty_like(rows)
    kv.kv_op_cache_read(cache, 0, slots, back[0], back[1])
    assert float((back - rows).abs().max()) < 0.5
    q = torch.randn(1, 16, 128, device="cuda") * 0.3
    out, lse = torch.empty_like(q), torch.empty(1, 16, device="cuda")
    scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(1, 16, cache, n), dtype=torch.uint8, device="cuda")
    kv.kv_op_paged_attention_batched(q, cache, 0, table, torch.tensor([n], dtype=torch.int32, device="cuda"), n, out,
                                     scratch, lse=lse)
    o, ls, size, most = S.attend(_np(q)[0], _np(back[0]), _np(back[1]), 128 ** -0.5)
    share = most * 2.0 ** -13 + 2.0 ** -14 + 102 * 2.0 ** -22
    assert (np.abs(_np(out)[0] - o) <= size * share).all()


def test_attention_same_bits_every_time_and_matches_the_single_request_operator(kv, torch):
    b = Batch(kv, torch, [1200, 40, 0, 513], 2, 4, 128, 16, 2, torch.float32)
    b.run(kv)
    first = (b.out.clone(), b.lse.clone())
    for _ in range(5):
        b.scratch.fill_(0xFF)
        b.run(kv)
        assert torch.equal(b.out, first[0]) and torch.equal(b.lse, first[1])
    for r in (0, 1, 3):
        n = b.lens[r]
        scratch = torch.empty(kv.kv_paged_attention_scratch_bytes(8, 128, n), dtype=torch.uint8, device="cuda")
        one = torch.empty(8, 128, device="cuda")
        kv.kv_op_paged_attention(b.q[r].contiguous(), b.cache, 0, b.table[r].contiguous(), n, scratch, one)
        assert float((one - b.out[r]).abs().max()) < 1e-4


# ------------------------------------------------------------------ streams, graphs, the operators together
def test_captured_graphs_replay_with_new_lists_and_share_scratch(kv, torch):
    b = Batch(kv, torch, [600, 90, 700], 2, 4, 64, 16, 1, torch.float32)
    c = Batch(kv, torch, [900, 1], 2, 4, 64, 16, 2, torch.float32, seed=1)
    need = max(b.scratch.numel(), c.scratch.numel())
    b.scratch = c.scratch = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    b.run(kv); c.run(kv)
    torch.cuda.synchronize()
    graphs = []
    for x in (b, c):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            x.run(kv)
        graphs.append(g)
    for lens in ([600, 90, 700], [1, 0, 650], [599, 64, 3]):
        b.lens_dev.copy_(torch.tensor(lens, dtype=torch.int32))
        b.out.fill_(7); c.out.fill_(7)
        for g in (graphs[0], graphs[1], graphs[1], graphs[0]):
            g.replay()
        torch.cuda.synchronize()
        b.check(torch, lens=lens)
        c.check(torch)


def test_operators_on_a_side_stream(kv, torch):
    b = Batch(kv, torch, [600, 90, 700], 2, 4, 64, 16, 1, torch.float32)
    b.run(kv)
    want = b.out.clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for how in (dict(stream=side), dict()):
        b.out.fill_(7)
        side.wait_stream(torch.cuda.current_stream())
        if how:
            b.run(kv, **how)
        else:
            with torch.cuda.stream(side):
                b.run(kv)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(b.out, want)


@pytest.mark.parametrize("elem", [1, 2])
@pytest.mark.parametrize("wire_layout", [0, 1])
def test_a_batch_migrates_and_decodes(kv, torch, elem, wire_layout):
    """Rotated K and V of three requests into the source's pages, the pages through pack and unpack into other blocks of
    a target cache, and one decode step there: rotate, append, attend.  Against the oracle on the same inputs."""
    shape = _shape(2, 64, 16, layers=2)
    lens, hq, d = [37, 16, 70], 8, 64
    rng = np.random.default_rng(9)
    rope = kv.Rope(32, layout="interleaved", base=1e4)
    source, target = (kv.PagedCache(shape, 16, elem_bytes=elem, fill=0) for _ in range(2))
    order, dest = rng.permutation(16), rng.permutation(16)
    at, tables = 0, []
    stored = []
    for r, n in enumerate(lens):
        need = -(-n // 16)
        tables.append(order[at:at + need])
        at += need
        for layer in range(2):
            qkv = torch.from_numpy(rng.standard_normal((n, hq + 4, d)).astype(np.float32)).cuda().to(torch.bfloat16)
            pos = torch.arange(n, device="cuda", dtype=torch.int32)
            k = torch.empty(n, 2, d, dtype=torch.bfloat16, device="cuda")
            kv.kv_op_rope(rope, qkv[:, hq:hq + 2], pos, k)
            slots = torch.from_numpy(tables[r][np.arange(n) // 16] * 16 + np.arange(n) % 16).cuda()
            kv.kv_op_cache_write(source, layer, k, qkv[:, hq + 2:], slots)
            stored.append((r, layer, k, qkv[:, hq + 2:]))
    blocks = np.concatenate(tables)
    wire = torch.zeros(len(blocks) * 2 * 2 * source.page_bytes, dtype=torch.uint8, device="cuda")
    kv.kv_pack_blocks(source, blocks, wire, wire_layout=wire_layout)
    merged = kv.kv_unpack_assemble(target, wire, np.arange(len(blocks)), dest[:len(blocks)], [], len(blocks) * 16,
                                   wire_layout=wire_layout)
    src, dst = _pages_numpy(source), _pages_numpy(target)
    assert np.array_equal(src[:, :, blocks], dst[:, :, merged])
    # one more token per request on the target; request 1 opens a block
    cols = 6
    table = np.full((3, cols), -1, dtype=np.int32)
    at = 0
    for r, t in enumerate(tables):
        table[r, :len(t)] = merged[at:at + len(t)]
        at += len(t)
    table[1, 1] = dest[len(blocks)]
    table = torch.from_numpy(table).cuda()
    for layer in range(2):
        qkv = torch.from_numpy(rng.standard_normal((3, hq + 4, d)).astype(np.float32)).cuda().to(torch.bfloat16)
        pos = torch.tensor(lens, dtype=torch.int32, device="cuda")
        fresh = qkv[:, hq:hq + 2].clone()
        kv.kv_op_rope(rope, qkv[:, :hq + 2], pos, qkv[:, :hq + 2])
        slots = table.gather(1, (pos // 16).long()[:, None])[:, 0].long() * 16 + pos % 16
        kv.kv_op_cache_write(target, layer, qkv[:, hq:hq + 2], qkv[:, hq + 2:], slots)
        q = qkv[:, :hq]
        out, lse = torch.empty(3, hq, d, dtype=torch.bfloat16, device="cuda"), torch.empty(3, hq, device="cuda")
        scratch = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(3, hq, target, cols * 16), dtype=torch.uint8, device="cuda")
        kv.kv_op_paged_attention_batched(q, target, layer, table, pos + 1, cols * 16, out, scratch, lse=lse)
        turned = S.rope(_np(fresh), lens, rope.frequencies(), "interleaved")
        assert np.abs(turned - _np(qkv[:, hq:hq + 2])).max() <= 2.0 ** -8 * np.abs(turned).max() * 1.01
        for r, n in enumerate(lens):
            k, v = next((k, v) for rr, l, k, v in stored if (rr, l) == (r, layer))
            k, v = torch.cat([k, qkv[r:r + 1, hq:hq + 2]]), torch.cat([v, qkv[r:r + 1, hq + 2:]])
            ks, vs = _np(k), _np(v)
            if elem == 1:
                t8 = S.e4m3_values()
                for x in (ks, vs):
                    for i in range(n + 1):
                        for h in range(2):
                            codes, byte = S.quantise_row(x[i, h])
                            x[i, h] = t8[codes] * 2.0 ** (byte - 127)
            o, ls, size, most = S.attend(_np(q)[r], ks, vs, d ** -0.5)
            share = most * 2.0 ** -13 + 2.0 ** -14 + (n / 16 + 64) * 2.0 ** -22
            assert (np.abs(_np(out)[r] - o) <= size * share + 2.0 ** -8 * np.abs(o) * 1.01).all()
            assert (np.abs(_np(lse)[r] - ls) <= share + 2.0 ** -23 * np.abs(ls)).all()


@pytest.mark.parametrize("lens", [[300, 20], [3000, 0, 900], [40] * 150])
def test_attention_in_place_of_its_queries(kv, torch, lens):
    b = Batch(kv, torch, lens, 4, 12, 64, 16, 1, torch.bfloat16)
    b.run(kv)
    want = b.out.clone()
    b.out = b.q
    b.run(kv)
    assert torch.equal(b.out, want)


def test_two_calls_at_once(kv, torch):
    """Two batches on two streams at the same time, each with scratch of its own, over and over."""
    a = Batch(kv, torch, [3000, 90, 700], 8, 8, 128, 16, 1, torch.bfloat16)
    b = Batch(kv, torch, [2500, 1, 0, 1800], 8, 4, 128, 16, 2, torch.float32, seed=2)
    a.run(kv); b.run(kv)
    torch.cuda.synchronize()
    want = a.out.clone(), b.out.clone()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(30):
        a.run(kv, stream=streams[0])
        b.run(kv, stream=streams[1])
    torch.cuda.synchronize()
    assert torch.equal(a.out, want[0]) and torch.equal(b.out, want[1])


@pytest.mark.parametrize("case", [(8, 128, 16), (3, 64, 7), (8, 128, 64), (2, 64, 16), (1, 64, 4)], ids=str)
def test_e4m3_pages_travel_whole(kv, torch, case):
    """Pack and unpack of e4m3 pages (one piece, several equal ones, a short one), scale bytes and padding included."""
    hkv, d, block = case
    shape = _shape(hkv, d, block, layers=2)
    for layout in ("layer_major", "block_major"):
        src, dst = (kv.PagedCache(shape, 13, layout=layout, elem_bytes=1) for _ in range(2))
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
        assert np.array_equal(wire[:src.page_bytes].cpu().numpy(), a[0, 0, 7])


def test_e4m3_suffix_streams_to_the_target(kv, torch):
    """Suffix streaming of an 8-bit cache: blocks are packed as they complete, the target's pages equal the source's."""
    from paper_2608_16477_b200 import streaming
    shape = _shape(2, 64, 16, layers=2)
    src, tgt = (kv.PagedCache(shape, 20, elem_bytes=1, fill=0) for _ in range(2))
    perm, fresh = np.random.default_rng(3).permutation(20), np.random.default_rng(4).permutation(20)
    k, n = 32, 32 + 53
    table = perm[:-(-n // 16)]
    rx = streaming.SuffixReceiver(tgt, request_id=1, expected_epoch=2, k_split=k, max_suffix_blocks=6, fresh_block_ids=fresh[2:10])
    tx = streaming.SuffixStreamer(src, table, k, request_id=1, epoch=2, transport=streaming.LoopbackTransport(rx))
    for pos in range(n):
        rows = torch.randn(2, 1, 2, 64, device="cuda")
        slots = torch.tensor([int(table[pos // 16]) * 16 + pos % 16], device="cuda")
        for layer in range(2):
            kv.kv_op_cache_write(src, layer, rows[0], rows[1] + layer, slots)
        if pos >= k:
            tx.on_token(pos)
            if pos % 20 == 0:
                tx.pump(max_blocks=1)
    tx.final_sync(n)
    merged = rx.assemble(fresh[:2], n, epoch=2)
    torch.cuda.synchronize()
    a, b = _pages_numpy(src), _pages_numpy(tgt)
    assert np.array_equal(a[:, :, table[2:]], b[:, :, merged[2:]]) and a[:, :, table[2:]].any()


def test_one_scratch_for_batches_of_every_size(kv, torch):
    """Scratch for the largest batch serves smaller ones, whatever path they take."""
    need, cases = 0, [([600] * 3, 1), ([700] * 9, 2), ([400], 2), ([800, 5] * 60, 1), ([30] * 120, 2)]
    batches = [Batch(kv, torch, lens, 8, 2, 64, 16, elem, torch.float32, ctx=800) for lens, elem in cases]
    need = kv.kv_paged_attention_batched_scratch_bytes(120, 16, batches[0].cache, 800)
    scratch = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")
    for b in batches:
        for ctx in (800, max(b.lens)):
            b.scratch, b.ctx = scratch, ctx
            b.run(kv)
            b.check(torch)
