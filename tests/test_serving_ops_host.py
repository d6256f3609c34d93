"""The batch-serving operators without a GPU: the oracle's pins, refusals of the C ABI (fake addresses are never
dereferenced) and of the binding, page sizes, rotary frequencies."""
import ctypes as C
import math

import numpy as np
import pytest

import synth
from oracle import kv_oracle as O
from oracle import serving_oracle as S


@pytest.fixture(scope="module")
def kv():
    import paper_2608_16477_b200 as kv
    kv.load()
    return kv


# ------------------------------------------------------------------ pins of the oracle
def test_e4m3_table_is_the_library_type():
    torch = pytest.importorskip("torch")
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    got = S.e4m3_values()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)])


def test_quantised_rows_round_like_the_library_cast():
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(5)
    for k in range(40):
        x = (rng.standard_normal(64) * 2.0 ** rng.integers(-20, 20)).astype(np.float32)
        codes, byte = S.quantise_row(x)
        e = byte - 127
        assert np.abs(x).max() <= 448 * 2.0 ** e and np.abs(x).max() > 448 * 2.0 ** (e - 1)
        want = torch.from_numpy(x.astype(np.float64) * 2.0 ** -e).float().to(torch.float8_e4m3fn).view(torch.uint8)
        assert np.array_equal(codes, want.numpy())


def test_quantise_row_corner_values():
    codes, byte = S.quantise_row(np.zeros(16))
    assert byte == 127 + S.MIN_EXP and not codes.any()
    codes, byte = S.quantise_row([448.0, -448.0, 1.0, 0.0])
    assert byte == 127 and list(codes[:2]) == [0x7E, 0xFE]
    _, byte = S.quantise_row([449.0, 1.0])
    assert byte == 128                                       # just above: the next power of two
    codes, byte = S.quantise_row([math.inf, -math.inf, math.nan, 2.0])
    assert byte == 127 - 7 and list(codes[:3]) == [S.NAN_CODE] * 3      # 2 = 256 * 2^-7
    codes, byte = S.quantise_row([3.4e38, -1.0])
    assert byte == 127 + S.MAX_EXP and codes[0] == 0x7E      # saturates


def test_rope_oracle_is_complex_multiplication_and_its_backward_the_transpose():
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 3, 2, 8))
    theta = S.rope_frequencies(6, 1e4)
    pos = [0, 5, -7]
    z = S.rope(x, pos, theta, "interleaved", gain=1.3)
    w = (x[..., 0:6:2] + 1j * x[..., 1:6:2]) * np.exp(1j * np.array(pos)[:, None, None] * theta) * 1.3
    assert np.allclose(z[..., 0:6:2], w.real) and np.allclose(z[..., 1:6:2], w.imag)
    assert np.array_equal(z[..., 6:], x[..., 6:])
    for layout in ("half", "interleaved"):
        a = S.rope(x, pos, theta, layout, 1.3)
        b = S.rope(y, pos, theta, layout, 1.3, backward=True)
        assert np.isclose((a[..., :6] * y[..., :6]).sum(), (x[..., :6] * b[..., :6]).sum())


def test_attend_oracle_equals_the_decode_oracle():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal((4, 64)), rng.standard_normal((9, 2, 64)), rng.standard_normal((9, 2, 64))
    out, lse, size, most = S.attend(q, k, v, 0.125)
    for h in range(4):
        s = np.array([q[h] @ k[n, h // 2] * 0.125 for n in range(9)])
        p = np.exp(s) / np.exp(s).sum()
        assert np.allclose(out[h], sum(p[n] * v[n, h // 2] for n in range(9)))
        assert np.isclose(lse[h], np.log(np.exp(s).sum()))
    assert (size >= np.abs(out) - 1e-12).all() and most > 0


# ------------------------------------------------------------------ pages and frequencies
def test_page_bytes(kv):
    assert kv.kv_cache_page_bytes(16, 8, 128, 2) == 32768 == synth.kv_page_bytes(synth.SHAPES["32b"])
    assert kv.kv_cache_page_bytes(16, 8, 128, 1) == 16384 + 128
    assert kv.kv_cache_page_bytes(7, 3, 64, 1) == 7 * 3 * 64 + 32        # 21 scale bytes, padded to 32
    for bad in ((0, 8, 128, 1), (16, 0, 128, 1), (16, 8, 0, 2)):
        with pytest.raises(kv.KVError) as e:
            kv.kv_cache_page_bytes(*bad)
        assert e.value.status == O.ERR_ARG
    with pytest.raises(kv.KVError) as e:
        kv.kv_cache_page_bytes(16, 8, 128, 4)
    assert e.value.status == O.ERR_SHAPE


def test_paged_cache_geometry_and_given_memory(kv):
    torch = pytest.importorskip("torch")
    s = synth.SHAPES["tiny"]
    for layout in ("layer_major", "block_major"):
        c = kv.PagedCache(s, 5, layout=layout, device="cpu", elem_bytes=1, fill=3)
        assert c.page_bytes == kv.kv_cache_page_bytes(16, 2, 64, 1) and c.data.dtype == torch.uint8
        assert c.data.numel() == 2 * 2 * 5 * c.page_bytes and c.desc.elem_bytes == 1
        again = kv.PagedCache(s, 5, layout=layout, device="cpu", elem_bytes=1, data=c.data)
        assert again.data.data_ptr() == c.data.data_ptr() == again.desc.base_dev
        assert again.pages([4, 0]).shape == (2, 2, 2, c.page_bytes)
    with pytest.raises(ValueError):
        kv.PagedCache(s, 6, device="cpu", elem_bytes=1, data=c.data)
    with pytest.raises(ValueError):
        kv.PagedCache(s, 6, device="cpu", elem_bytes=3)
    with pytest.raises(ValueError):
        c.as_logical_numpy()


@pytest.mark.parametrize("kw", [dict(), dict(scaling="linear", factor=4.0), dict(scaling="ntk", factor=8.0),
                                dict(scaling="parts", factor=8.0, original_ctx=4096, low=1.0, high=32.0),
                                dict(scaling="parts", factor=32.0, original_ctx=8192, low=1.0, high=4.0)])
@pytest.mark.parametrize("rotary", [4, 50, 64, 128, 256])
def test_rope_frequencies(kv, kw, rotary):
    got = kv.Rope(rotary, base=1e6, **kw).frequencies()
    want = S.rope_frequencies(rotary, 1e6, kw.get("scaling", "none"), kw.get("factor", 1.0), kw.get("original_ctx", 0.0),
                              kw.get("low", 1.0), kw.get("high", 32.0))
    assert np.abs(got / want - 1).max() < 1e-13


def test_rope_plan_refusals(kv):
    def status(*a, **k):
        with pytest.raises(kv.KVError) as e:
            kv.Rope(*a, **k)
        return e.value.status
    for rotary in (0, -2, 7, 258):
        assert status(rotary) == O.ERR_SHAPE
    for base in (0.0, -1.0, math.inf, math.nan, 0.5):         # 0.5: pairs that turn by more than a radian a position
        assert status(64, base=base) == O.ERR_ARG
    assert status(64, gain=0.0) == O.ERR_ARG
    assert status(64, scaling="linear", factor=0.0) == status(64, scaling="linear", factor=0.5) == O.ERR_ARG
    assert status(2, scaling="ntk", factor=2.0) == O.ERR_SHAPE
    assert status(64, scaling="parts", factor=2.0, original_ctx=0.0) == O.ERR_ARG
    assert status(64, scaling="parts", factor=2.0, original_ctx=10.0, low=4.0, high=4.0) == O.ERR_ARG
    for bad in (dict(layout="other"), dict(scaling="other")):
        with pytest.raises(ValueError):
            kv.Rope(64, **bad)
    lib = kv.load()
    assert lib.kv_rope_create(None, C.byref(C.c_void_p())) == O.ERR_ARG
    r = kv.Rope(64)
    buf = (C.c_double * 31)()
    assert lib.kv_rope_frequencies(r.handle, buf, 31) == O.ERR_ARG


# ------------------------------------------------------------------ refusals of the operators
FAKE = 0x7000000000


def _desc(**kw):
    from paper_2608_16477_b200.binding import CacheDesc
    f = dict(base_dev=FAKE, num_blocks=16, block_size=16, n_layers=2, n_kv_heads=2, head_dim=128, elem_bytes=1)
    f.update({k: v for k, v in kw.items() if k in f})
    page = f["block_size"] * f["n_kv_heads"] * f["head_dim"] * f["elem_bytes"] + \
        (-(-f["block_size"] * f["n_kv_heads"] // 16) * 16 if f["elem_bytes"] == 1 else 0)
    f.update(layer_stride=2 * 16 * page, kv_stride=16 * page, block_stride=page)
    f.update(kw)
    return CacheDesc(*[f[n] for n, _ in CacheDesc._fields_])


def test_rope_refusals(kv):
    lib, r = kv.load(), kv.Rope(64)
    x, out, pos = FAKE, FAKE + 0x1000000, FAKE + 0x2000000

    def call(x=x, xt=512, xh=128, dtype=0, t=4, h=4, d=128, pos=pos, out=out, ot=512, oh=128, rope=r.handle):
        return lib.kv_op_rope(rope, x, xt, xh, dtype, t, h, d, pos, 0, out, ot, oh, 0)
    assert call(t=0) == O.OK
    assert call(rope=None) == call(x=None) == call(out=None) == call(pos=None) == O.ERR_ARG
    assert call(t=-1) == call(h=0) == call(dtype=2) == call(dtype=-1) == O.ERR_ARG
    assert call(d=62) == call(d=1025) == O.ERR_SHAPE
    assert call(x=x + 1) == call(out=out + 1) == call(pos=pos + 2) == call(dtype=1, x=x + 2) == O.ERR_ARG
    assert call(xt=-1) == call(oh=127) == call(ot=127) == O.ERR_ARG
    assert call(ot=128, oh=128) == O.ERR_ARG                  # tokens and heads of the output overlap
    assert call(ot=128, oh=511) == O.ERR_ARG                  # head-major, one element short
    assert call(out=x, ot=640) == O.ERR_ARG                   # in place with other strides


@pytest.mark.parametrize("elem", [1, 2])
def test_row_refusals(kv, elem):
    lib = kv.load()
    k, v, slots = FAKE + 0x1000000, FAKE + 0x2000000, FAKE + 0x3000000
    good = _desc(elem_bytes=elem)

    def both(desc=good, layer=0, k=k, kt=256, kh=128, v=v, vt=256, vh=128, dtype=0, t=5, slots=slots):
        a = lib.kv_op_cache_write(C.byref(desc), layer, k, kt, kh, v, vt, vh, dtype, t, slots, 0)
        b = lib.kv_op_cache_read(C.byref(desc), layer, slots, t, k, kt, kh, v, vt, vh, dtype, 0)
        return a, b
    arg, shape = (O.ERR_ARG,) * 2, (O.ERR_SHAPE,) * 2
    assert both(t=0) == (O.OK, O.OK)
    assert both(t=-1) == both(dtype=3) == both(k=None) == both(v=None) == both(slots=None) == arg
    assert both(layer=2) == both(layer=-1) == both(desc=_desc(elem_bytes=elem, head_dim=96)) == shape
    assert both(desc=_desc(elem_bytes=4)) == shape
    assert both(k=k + 8) == both(v=v + 2) == both(slots=slots + 4) == arg
    assert both(kt=260) == both(vh=132) == both(kt=-256) == arg
    assert both(desc=_desc(elem_bytes=elem, block_stride=16)) == arg
    assert both(desc=_desc(elem_bytes=elem, base_dev=FAKE + 8)) == arg
    # rows that are written may not overlap; rows that are read may (a broadcast)
    assert both(kh=0, t=0) == (O.OK, O.OK)
    assert lib.kv_op_cache_read(C.byref(good), 0, slots, 5, k, 256, 0, v, 256, 128, 0, 0) == O.ERR_ARG
    assert lib.kv_op_cache_read(C.byref(good), 0, slots, 5, k, 0, 128, v, 256, 128, 0, 0) == O.ERR_ARG
    assert lib.kv_op_cache_read(C.byref(good), 0, slots, 5, k, 128, 128, v, 256, 128, 0, 0) == O.ERR_ARG
    assert lib.kv_op_cache_read(C.byref(good), 0, slots, 5, k, 128, 632, v, 256, 128, 0, 0) == O.ERR_ARG


@pytest.mark.parametrize("elem", [1, 2])
def test_batched_attention_refusals(kv, elem):
    lib = kv.load()
    q, tab, lens, scr, out, lse = (FAKE + i * 0x1000000 for i in range(1, 7))
    need = lib.kv_paged_attention_batched_scratch_bytes(3, 8, 2, 128, 4096)
    assert need > 0

    def call(q=q, qs=1024, dtype=0, r=3, hq=8, desc=_desc(elem_bytes=elem), layer=0, tab=tab, ts=256, lens=lens, ctx=4096,
             scale=0.1, scr=scr, need=need, out=out, os=1024, lse=lse):
        return lib.kv_op_paged_attention_batched(q, qs, dtype, r, hq, C.byref(desc), layer, tab, ts, lens, ctx, scale,
                                                 scr, need, out, os, lse, 0)
    assert call(r=0) == O.OK
    assert call(r=-1) == call(hq=0) == call(ctx=0) == call(dtype=2) == O.ERR_ARG
    for p in ("q", "tab", "lens", "out"):
        assert call(**{p: None}) == O.ERR_ARG
    for s in (0.0, -1.0, math.inf, math.nan, 3e38):
        assert call(scale=s) == O.ERR_ARG
    assert call(q=q + 8) == call(out=out + 8) == call(tab=tab + 2) == call(lens=lens + 1) == call(lse=lse + 2) == O.ERR_ARG
    assert call(qs=1020) == call(os=1020) == call(os=1016) == call(qs=-1024) == call(ts=-1) == O.ERR_ARG
    assert call(hq=7) == call(layer=2) == call(layer=-1) == call(desc=_desc(head_dim=96)) == O.ERR_SHAPE
    assert call(desc=_desc(elem_bytes=4)) == call(ctx=(1 << 26) + 1) == O.ERR_SHAPE
    assert call(ts=255) == O.ERR_TABLE_SHORT
    assert call(scr=None) == call(scr=scr + 8) == call(need=need - 1) == O.ERR_WORKSPACE
    assert lib.kv_paged_attention_batched_scratch_bytes(3, 8, 3, 128, 4096) == O.ERR_SHAPE
    assert lib.kv_paged_attention_batched_scratch_bytes(3, 8, 2, 96, 4096) == O.ERR_SHAPE
    assert lib.kv_paged_attention_batched_scratch_bytes(-1, 8, 2, 128, 4096) == O.ERR_ARG
    assert lib.kv_paged_attention_batched_scratch_bytes(3, 8, 2, 128, 0) == O.ERR_ARG


@pytest.mark.parametrize("heads", [(64, 8), (8, 1), (4, 2), (40, 5), (256, 4)])
def test_scratch_for_a_batch_serves_every_smaller_one(kv, heads):
    """The size grows with the requests and the context; a smaller call on a larger call's scratch is not refused (the fake
    addresses get as far as the missing device)."""
    lib = kv.load()
    hq, hkv = heads
    for d in (64, 128):
        for ctx in (1, 384, 385, 500, 512, 513, 768, 769, 5000):
            sizes = [lib.kv_paged_attention_batched_scratch_bytes(r, hq, hkv, d, ctx) for r in (0, 1, 2, 7, 8, 9, 40, 100, 700)]
            assert sizes == sorted(sizes) and sizes[0] > 0
        for r in (1, 7, 8, 100):
            sizes = [lib.kv_paged_attention_batched_scratch_bytes(r, hq, hkv, d, c) for c in (1, 384, 385, 512, 768, 769, 9000)]
            assert sizes == sorted(sizes)
    import torch
    if torch.cuda.is_available():
        return
    need = lib.kv_paged_attention_batched_scratch_bytes(100, hq, hkv, 128, 4096)
    q, tab, lens, scr, out = (FAKE + i * 0x1000000 for i in range(1, 6))
    for elem in (1, 2):
        desc = _desc(elem_bytes=elem, n_kv_heads=hkv)
        for r in (1, 5, 8, 60, 100):
            for ctx in (100, 390, 600, 800, 4096):
                got = lib.kv_op_paged_attention_batched(q, hq * 128, 0, r, hq, C.byref(desc), 0, tab, 256, lens, ctx, 0.1,
                                                        scr, need, out, hq * 128, None, 0)
                assert got == -13, (r, ctx, got)


def test_entry_points_for_bf16_pages_refuse_e4m3_pages(kv):
    lib, d = kv.load(), _desc()
    tab, q, out, scr = FAKE + 0x1000000, FAKE + 0x2000000, FAKE + 0x3000000, FAKE + 0x4000000
    assert lib.kv_op_paged_attention(q, 8, C.byref(d), 0, tab, 100, scr, 1 << 20, out, 0) == O.ERR_SHAPE
    assert lib.kv_op_paged_attention_noalloc(q, 8, C.byref(d), 0, tab, 100, out, 0) == O.ERR_SHAPE
    assert lib.kv_op_attention_prefill(q, 10, 16, 8, 2, 128, C.byref(d), 0, tab, out, None, 0) == O.ERR_SHAPE
    # pack knows them: a wire one byte short of the pages with their scales is refused as short
    ids = (C.c_int32 * 2)(1, 2)
    page = kv.kv_cache_page_bytes(16, 2, 128, 1)
    assert lib.kv_pack_blocks(C.byref(d), ids, 2, scr, 2 * 2 * 2 * page - 1, 0, 0) == O.ERR_WIRE_SIZE


def test_binding_refuses_what_does_not_fit(kv):
    torch = pytest.importorskip("torch")
    s = synth.SHAPES["tiny"]
    cache = kv.PagedCache(s, 4, device="cpu", elem_bytes=1)
    rope = kv.Rope(64)
    x, pos = torch.zeros(3, 4, 64), torch.zeros(3, dtype=torch.int32)
    bad = [lambda: kv.kv_op_rope(rope, x[0], pos, x[0]),
           lambda: kv.kv_op_rope(rope, x, pos, x.bfloat16()),
           lambda: kv.kv_op_rope(rope, x, pos.long(), x),
           lambda: kv.kv_op_rope(rope, x, pos.float(), x),
           lambda: kv.kv_op_rope(rope, x, pos[:2], x),
           lambda: kv.kv_op_rope(rope, x.half(), pos, x.half()),
           lambda: kv.kv_op_rope(rope, x.transpose(1, 2), pos, x.transpose(1, 2)),
           lambda: kv.kv_op_rope(rope, x, pos, x)]                                  # not on a CUDA device
    rows, slots = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int64)
    bad += [lambda: kv.kv_op_cache_write(cache, 0, rows, rows, slots.int()),
            lambda: kv.kv_op_cache_write(cache, 0, rows, rows, slots.double()),
            lambda: kv.kv_op_cache_write(cache, 0, rows, rows[:2], slots),
            lambda: kv.kv_op_cache_write(cache, 0, rows, rows.bfloat16(), slots),
            lambda: kv.kv_op_cache_write(cache, 0, rows[:, :1], rows[:, :1], slots),
            lambda: kv.kv_op_cache_read(cache, 0, slots[:, None], rows, rows),
            lambda: kv.kv_op_cache_read(cache, 0, slots, rows.double(), rows.double())]
    q, tab, lens = torch.zeros(2, 4, 64), torch.zeros(2, 4, dtype=torch.int32), torch.ones(2, dtype=torch.int32)

    def attend(q=q, tab=tab, lens=lens, out=q, lse=None, ctx=64):
        return lambda: kv.kv_op_paged_attention_batched(q, cache, 0, tab, lens, ctx, out, None, lse=lse)
    bad += [attend(q=q[..., :32]), attend(out=q[:1]), attend(out=q.bfloat16()), attend(tab=tab.long()), attend(tab=tab[0]),
            attend(tab=tab[:1]), attend(lens=lens.long()), attend(lens=lens[:1]), attend(lse=torch.zeros(2, 3)),
            attend(lse=torch.zeros(2, 4, dtype=torch.float64)), attend(q=q[:, ::2]), attend(tab=tab.t()),
            attend(tab=torch.zeros(4, dtype=torch.int32).expand(2, 4))]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    with pytest.raises(kv.KVError) as e:
        attend(ctx=65)()
    assert e.value.status == O.ERR_TABLE_SHORT
