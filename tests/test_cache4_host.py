"""A cache in four bits and the selection of blocks without a GPU: the oracle's pins, page sizes, refusals of the C ABI (fake addresses
are never dereferenced) and of the binding, sizes of scratch."""
import ctypes as C
import math

import numpy as np
import pytest

import synth
from oracle import kv_oracle as O
from oracle import pages4_oracle as P

E2M1 = -2
CLOSED = -13                      # as far as a call on fake addresses gets without a device
FAKE = 0x7000000000


def _at(i):
    return FAKE + i * 0x1000000


@pytest.fixture(scope="module")
def kv():
    import paper_2608_16477_b200 as kv
    kv.load()
    return kv


@pytest.fixture
def no_gpu():
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")


# ------------------------------------------------------------------ pins of the oracle
def test_codes_are_a_sign_two_exponent_bits_and_one_more():
    for code, value in enumerate(P.e2m1_values()):
        exponent, part = (code >> 1) & 3, code & 1
        want = (1 + part / 2) * 2.0 ** (exponent - 1) if exponent else part / 2
        assert value == (-want if code & 8 else want)


def test_rows_at_the_borders_of_the_scales():
    codes, groups, byte = P.quantise_row(np.zeros(32))
    assert byte == 127 + P.MIN_EXP and not codes.any() and list(groups) == [1, 1]
    row = np.zeros(16)
    row[:9] = [2688.0, 5.0 * 448, 3.5 * 448, 2.5 * 448, 1.75 * 448, 1.25 * 448, 0.75 * 448, 0.25 * 448, -0.25 * 448]
    codes, groups, byte = P.quantise_row(row)
    assert byte == 127 and groups[0] == 0x7E
    assert list(codes[:9]) == [7, 7, 6, 5, 4, 3, 2, 1, 9]              # halves go away from zero
    assert P.quantise_row(np.nextafter(row, 0))[0].tolist()[1:9] == [6, 5, 4, 3, 2, 1, 0, 8]
    row[0] = np.nextafter(2688.0, 3000)
    assert P.quantise_row(row)[2] == 128
    codes, groups, byte = P.quantise_row([1.0] * 15 + [math.inf] + [-6.0] + [0.0] * 14 + [-0.0])
    assert groups[0] == P.NAN_SCALE and not codes[:16].any() and codes[16] == 15 and codes[31] == 8
    assert byte == 127 - 8                                            # 6 <= 2688 * 2^-8 = 10.5
    assert P.quantise_row([3.4e38] + [0.0] * 15)[2] == 127 + P.MAX_EXP
    assert np.isfinite(P.stored([3.4e38] + [0.0] * 15)).all() and P.stored([3.4e38] + [0.0] * 15).max() < np.finfo(np.float32).max


def test_a_stored_value_is_off_by_half_a_step_at_most():
    """A group's scale s has max |x| <= 6 s and is at most an eighth above the least such number (e4m3 normals): the steps of the codes are
    s / 2 up to 2 s, s up to 4 s, 2 s up to 6 s."""
    rng = np.random.default_rng(3)
    for _ in range(30):
        x = rng.standard_normal(64) * 2.0 ** rng.integers(-9, 9, 64)
        codes, groups, byte = P.quantise_row(x)
        s = np.repeat(P.e4m3_values()[groups], 16) * 2.0 ** (byte - 127.0)
        a = np.abs(x) / s
        assert (a <= 6).all()
        step = np.where(a <= 2, 0.5, np.where(a <= 4, 1.0, 2.0)) * s
        assert (np.abs(P.stored(x) - x) <= step / 2).all()


def test_bounds_hold_the_keys_and_no_more_than_a_unit_beyond():
    rng = np.random.default_rng(4)
    keys = rng.standard_normal((16, 64)) * 2.0 ** rng.integers(-6, 6, 64)
    codes, byte = P.block_bounds(keys)
    unit = 2.0 ** (byte - 127)
    up, low = codes.astype(np.float64) * unit
    assert (up >= keys.max(0)).all() and (up < keys.max(0) + unit).all()
    assert (low <= keys.min(0)).all() and (low > keys.min(0) - unit).all()
    assert np.abs(keys).max() <= 127 * unit < 2 * np.abs(keys).max()
    assert P.block_bounds(np.zeros((2, 4)))[1] == 127 - 60
    assert P.block_bounds([[127.0, 0]])[1] == 127 and P.block_bounds([[127.5, 0]])[1] == 128
    for bad in (math.nan, math.inf, 127.1 * 2.0 ** 60):
        codes, byte = P.block_bounds([[1.0, bad]])
        assert byte == P.INFINITE and not codes.any()


def test_the_score_is_no_less_than_any_sum_over_the_heads():
    """Up to the rounding of the query's code: half a unit for each of the 2 d numbers, times bounds of 127 units at most."""
    rng = np.random.default_rng(5)
    for _ in range(20):
        q, keys = rng.standard_normal((4, 64)), rng.standard_normal((16, 64))
        codes, byte = P.block_bounds(keys)
        u = P.query_code(q)
        assert np.abs(u).max() > 16383
        unit = np.maximum(q, 0).sum(0).max() / u[:64].max()
        score = int(codes.astype(np.int64).reshape(-1) @ u) * 2.0 ** (byte - 127) * 2.0 ** np.round(np.log2(unit))
        room = 0.5 * 2.0 ** np.round(np.log2(unit)) * np.abs(codes.astype(float)).sum() * 2.0 ** (byte - 127)
        assert score >= max((q @ k).sum() for k in keys) - room


def test_selection_keeps_the_ends_and_the_first_of_equals():
    codes, scales = np.ones((10, 2, 4), np.int8), np.full(10, 127, np.uint8)
    q, table = np.ones((2, 4)), np.arange(10)[::-1].copy()
    assert P.select(q, codes, scales, table, 150, 16, 10, 1, 2) == (list(range(10)), 150)
    assert P.select(q, codes, scales, table, 150, 16, 5, 1, 2) == ([0, 1, 2, 8, 9], 150 - 5 * 16)
    codes[table[6]] = 2
    assert P.select(q, codes, scales, table, 150, 16, 5, 1, 2) == ([0, 1, 6, 8, 9], 70)
    scales[table[7]] = P.INFINITE
    assert P.select(q, codes, scales, table, 145, 16, 4, 1, 2) == ([0, 7, 8, 9], 145 - 6 * 16)
    table[3] = -1
    assert P.select(q, codes, scales, table, 150, 16, 4, 1, 2)[0] == [0, 3, 8, 9]
    assert P.select(np.full((2, 4), math.nan), codes, scales, np.arange(10), 150, 16, 4, 1, 3)[0] == [0, 7, 8, 9]


# ------------------------------------------------------------------ sizes
def test_page_bytes(kv):
    assert kv.kv_cache_page_bytes(16, 8, 128, 0.5) == 8 * 16 * (64 + 8 + 1) == 9344
    assert kv.kv_cache_page_bytes(7, 3, 64, 0.5) == 3 * 272                # 7 * 37 = 259, padded
    assert kv.kv_cache_page_bytes(1, 1, 16, 0.5) == 16                     # 10, padded
    assert kv.kv_bytes_per_token(2, 3, 64, 0.5) == 2 * kv.load().kv_bytes_per_token(1, 3, 64, E2M1) == 2 * 2 * 3 * 32
    for bad in ((0, 8, 128, 0.5), (16, 0, 128, 0.5)):
        with pytest.raises(kv.KVError) as e:
            kv.kv_cache_page_bytes(*bad)
        assert e.value.status == O.ERR_ARG
    for bad in ((16, 8, 24, 0.5), (16, 8, 128, -1), (16, 8, 128, 0)):
        with pytest.raises(kv.KVError) as e:
            kv.kv_cache_page_bytes(*bad)
        assert e.value.status == O.ERR_SHAPE


def test_paged_cache_geometry_and_given_memory(kv):
    torch = pytest.importorskip("torch")
    s = synth.SHAPES["tiny"]
    for layout in ("layer_major", "block_major"):
        c = kv.PagedCache(s, 5, layout=layout, device="cpu", elem_bytes=0.5, fill=3)
        assert c.page_bytes == kv.kv_cache_page_bytes(16, 2, 64, 0.5) and c.data.dtype == torch.uint8
        assert c.data.numel() == 2 * 2 * 5 * c.page_bytes and c.desc.elem_bytes == E2M1
        again = kv.PagedCache(s, 5, layout=layout, device="cpu", elem_bytes=0.5, data=c.data)
        assert again.data.data_ptr() == c.data.data_ptr() == again.desc.base_dev
        assert again.pages([4, 0]).shape == (2, 2, 2, c.page_bytes)
        bounds = kv.BlockBounds(c)
        assert bounds.codes.shape == (2, 5, 2, 2, 64) and bounds.scales.shape == (2, 5, 2)
        assert kv.BlockBounds(c, bounds.codes, bounds.scales).codes.data_ptr() == bounds.codes.data_ptr()
        for bad in (dict(codes=bounds.codes[:1]), dict(codes=bounds.codes.byte()), dict(scales=bounds.scales.char()),
                    dict(scales=bounds.scales[..., :1]), dict(codes=bounds.codes.transpose(0, 1).contiguous().transpose(0, 1))):
            with pytest.raises(ValueError):
                kv.BlockBounds(c, **bad)
    with pytest.raises(ValueError):
        kv.PagedCache(s, 6, device="cpu", elem_bytes=0.5, data=c.data)
    with pytest.raises(ValueError):
        c.as_logical_numpy()


def test_selection_scratch_grows_with_requests_heads_and_context(kv):
    size = kv.load().kv_select_blocks_scratch_bytes
    assert size(0, 8, 16, 100) == 0
    for vary in (lambda x: size(x, 8, 16, 5000), lambda x: size(4, x, 16, 5000), lambda x: size(4, 8, 16, x)):
        sizes = [vary(x) for x in (1, 2, 7, 64, 700, 65535)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    assert size(65535, 65535, 1, 1 << 26) == 65535 * 65535 * (1 << 26) * 4         # past 32 bits
    assert size(-1, 8, 16, 5) == size(1, 0, 16, 5) == size(1, 8, 0, 5) == size(1, 8, 16, 0) == O.ERR_ARG
    assert size(1, 8, 16, (1 << 26) + 1) == O.ERR_SHAPE


# ------------------------------------------------------------------ refusals of the C entry points
def _desc(elem=E2M1, **kw):
    from paper_2608_16477_b200.binding import CacheDesc
    f = dict(base_dev=FAKE, num_blocks=16, block_size=16, n_layers=2, n_kv_heads=2, head_dim=128, elem_bytes=elem)
    f.update({k: v for k, v in kw.items() if k in f})
    rows = f["block_size"] * f["n_kv_heads"]
    page = {E2M1: f["n_kv_heads"] * (-(-f["block_size"] * (f["head_dim"] // 2 + f["head_dim"] // 16 + 1) // 16) * 16),
            1: rows * f["head_dim"] + -(-rows // 16) * 16, 2: rows * f["head_dim"] * 2}.get(elem, 1 << 16)
    f.update(layer_stride=2 * 16 * page, kv_stride=16 * page, block_stride=page)
    f.update(kw)
    return CacheDesc(*[f[n] for n, _ in CacheDesc._fields_])


def test_descriptors_of_e2m1_pages(kv):
    lib, slots = kv.load(), _at(3)

    def call(desc):
        return lib.kv_op_cache_write(C.byref(desc), 0, _at(1), 256, 128, _at(2), 256, 128, 0, 0, slots, 0)
    assert call(_desc()) == O.OK
    assert call(_desc(block_stride=9344 // 4 - 16)) == O.ERR_ARG                   # pages that overlap
    assert call(_desc(block_stride=9344 // 4)) == O.OK
    assert call(_desc(block_stride=9344 // 4 + 8)) == call(_desc(base_dev=FAKE + 4)) == O.ERR_ARG
    assert call(_desc(head_dim=120)) == call(_desc(elem=-1)) == call(_desc(elem=0)) == O.ERR_SHAPE


def test_entry_points_for_bf16_pages_refuse_e2m1_pages(kv):
    lib, d = kv.load(), _desc()
    tab, q, out, scr = (_at(i) for i in range(1, 5))
    assert lib.kv_op_paged_attention(q, 8, C.byref(d), 0, tab, 100, scr, 1 << 20, out, 0) == O.ERR_SHAPE
    assert lib.kv_op_paged_attention_noalloc(q, 8, C.byref(d), 0, tab, 100, out, 0) == O.ERR_SHAPE
    assert lib.kv_op_attention_prefill(q, 10, 16, 8, 2, 128, C.byref(d), 0, tab, out, None, 0) == O.ERR_SHAPE
    ids = (C.c_int32 * 2)(1, 2)
    page = kv.kv_cache_page_bytes(16, 2, 128, 0.5)
    assert lib.kv_pack_blocks(C.byref(d), ids, 2, scr, 2 * 2 * 2 * page - 1, 0, 0) == O.ERR_WIRE_SIZE


@pytest.mark.parametrize("elem", [E2M1, 1, 2])
def test_append_refusals(kv, elem, no_gpu):
    lib, rope, wide = kv.load(), kv.Rope(64), kv.Rope(256)
    k, v, q, out, pos, slots = (_at(i) for i in range(1, 7))
    good = _desc(elem)

    def call(rope=rope.handle, desc=good, layer=0, q=q, qt=512, qh=128, hq=4, out=out, ot=512, oh=128, k=k, kt=256, kh=128, v=v, vt=256,
             vh=128, dtype=0, t=5, pos=pos, slots=slots):
        return lib.kv_op_cache_append(rope, C.byref(desc) if desc else None, layer, q, qt, qh, hq, out, ot, oh, k, kt, kh, v, vt, vh, dtype, t,
                                      pos, slots, 0)
    assert call() == CLOSED and call(t=0) == O.OK
    assert call(rope=None) == call(desc=None) == call(t=-1) == call(hq=-1) == call(dtype=2) == O.ERR_ARG
    for p in ("k", "v", "q", "out", "pos", "slots"):
        assert call(**{p: None}) == O.ERR_ARG
        assert call(**{p: dict(k=k, v=v, q=q, out=out, pos=pos, slots=slots)[p] + 2}) == O.ERR_ARG
    assert call(hq=0, q=None, out=None, qt=-3, qh=1, ot=-3, oh=1) == CLOSED
    for s in ("kt", "kh", "vt", "vh", "qt", "qh", "ot", "oh"):
        assert call(**{s: -256}) == call(**{s: 516}) == O.ERR_ARG
    assert call(oh=64) == call(ot=128) == call(ot=448) == O.ERR_ARG               # outputs that overlap
    assert call(qt=0, kh=0, vt=0) == CLOSED                                       # inputs may
    assert call(out=q) == CLOSED and call(out=q, ot=640) == call(out=q, qh=0) == O.ERR_ARG
    assert call(rope=wide.handle) == call(layer=2) == call(layer=-1) == call(t=(1 << 30) + 1) == O.ERR_SHAPE
    assert call(desc=_desc(elem, head_dim=96)) == call(hq=1 << 20, ot=1 << 30) == O.ERR_SHAPE


@pytest.mark.parametrize("elem", [E2M1, 1, 2])
def test_bounds_refusals(kv, elem):
    lib = kv.load()
    blocks, counts, codes, scales = (_at(i) for i in range(1, 5))

    def call(desc=_desc(elem), layer=0, blocks=blocks, counts=counts, n=3, codes=codes, scales=scales):
        return lib.kv_op_block_bounds(C.byref(desc) if desc else None, layer, blocks, counts, n, codes, scales, 0)
    assert call(n=0) == O.OK
    assert call(n=-1) == call(desc=None) == O.ERR_ARG
    assert call(blocks=None) == call(counts=None) == call(codes=None) == call(scales=None) == O.ERR_ARG
    assert call(blocks=blocks + 2) == call(counts=counts + 1) == call(codes=codes + 8) == O.ERR_ARG
    assert call(layer=2) == call(layer=-1) == call(desc=_desc(elem, head_dim=96)) == O.ERR_SHAPE


def test_selection_refusals(kv, no_gpu):
    lib = kv.load()
    q, codes, scales, tab, lens, scr, kept, kept_lens = (_at(i) for i in range(1, 9))
    need = lib.kv_select_blocks_scratch_bytes(3, 2, 16, 4096)
    assert need == 3 * 2 * 256 * 4

    def call(q=q, qs=1024, dtype=0, r=3, hq=8, h=2, d=128, codes=codes, scales=scales, nb=500, block=16, tab=tab, ts=256, lens=lens, ctx=4096,
             first=1, last=2, keep=20, scr=scr, need=need, kept=kept, kept_lens=kept_lens):
        return lib.kv_op_select_blocks(q, qs, dtype, r, hq, h, d, codes, scales, nb, block, tab, ts, lens, ctx, first, last, keep, scr, need,
                                       kept, kept_lens, 0)
    assert call() == CLOSED and call(r=0) == O.OK
    assert call(r=-1) == call(hq=0) == call(h=0) == call(nb=0) == call(block=0) == call(ctx=0) == call(dtype=2) == O.ERR_ARG
    assert call(first=-1) == call(last=0) == call(keep=0) == call(first=18, last=3) == call(first=2 ** 31 - 1) == O.ERR_ARG
    assert call(first=18) == call(first=0, last=20) == call(keep=3) == CLOSED
    for p in ("q", "codes", "scales", "tab", "lens", "kept", "kept_lens"):
        assert call(**{p: None}) == O.ERR_ARG
    assert call(q=q + 8) == call(codes=codes + 8) == call(tab=tab + 2) == call(lens=lens + 2) == call(kept=kept + 1) == O.ERR_ARG
    assert call(kept_lens=kept_lens + 2) == call(qs=1020) == call(qs=-1024) == call(ts=-1) == O.ERR_ARG
    assert call(hq=7) == call(d=96) == call(ctx=(1 << 26) + 1) == call(r=65536) == call(h=65536, hq=65536) == O.ERR_SHAPE
    assert call(keep=(1 << 22) + 1) == O.ERR_SHAPE
    assert call(ts=255) == O.ERR_TABLE_SHORT
    assert call(scr=None) == call(scr=scr + 8) == call(need=need - 1) == O.ERR_WORKSPACE
    assert call(keep=256, scr=None, need=0) == CLOSED                             # nothing to choose
    more = lib.kv_select_blocks_scratch_bytes(40, 2, 16, 9000)
    for r in (1, 5, 40):
        for ctx in (1, 500, 9000):
            assert call(r=r, ctx=ctx, ts=600, need=more) == CLOSED


@pytest.mark.parametrize("elem", [E2M1, 1, 2])
def test_selected_attention_refusals(kv, elem, no_gpu):
    lib = kv.load()
    q, tab, lens, scr, out, lse = (_at(i) for i in range(1, 7))
    need = lib.kv_paged_attention_batched_scratch_bytes(3, 8, 2, 128, 1024)

    def call(q=q, qs=1024, dtype=0, r=3, hq=8, desc=_desc(elem), layer=0, tab=tab, ts=128, hs=64, lens=lens, most=1024, scale=0.1, scr=scr,
             need=need, out=out, os=1024, lse=lse):
        return lib.kv_op_paged_attention_selected(q, qs, dtype, r, hq, C.byref(desc), layer, tab, ts, hs, lens, most, scale, scr, need, out,
                                                  os, lse, 0)
    assert call() == CLOSED and call(r=0) == O.OK
    assert call(hs=0) == call(hs=-64) == call(ts=-1) == call(most=0) == call(dtype=3) == call(scale=math.nan) == O.ERR_ARG
    for p in ("q", "tab", "lens", "out"):
        assert call(**{p: None}) == O.ERR_ARG
    assert call(lse=None) == CLOSED
    assert call(out=q, os=2048) == call(os=1016) == call(qs=1020) == O.ERR_ARG
    assert call(ts=63) == call(hs=63) == O.ERR_TABLE_SHORT
    assert call(hq=7) == call(layer=2) == call(desc=_desc(elem, head_dim=96)) == O.ERR_SHAPE
    assert call(scr=None) == call(need=need - 1) == O.ERR_WORKSPACE


@pytest.mark.parametrize("heads", [(64, 8), (8, 1), (12, 3), (256, 4)])
@pytest.mark.parametrize("dtype", [0, 1])
def test_scratch_serves_every_smaller_batch_of_every_format(kv, heads, dtype, no_gpu):
    lib, (hq, hkv) = kv.load(), heads
    q, tab, lens, scr, out = (_at(i) for i in range(1, 6))
    ctxs, reqs = (300, 385, 513, 769, 1024, 1025, 4096), (1, 7, 8, 16, 60, 120, 700)
    for n in reqs:
        for ctx in ctxs:
            need = lib.kv_paged_attention_batched_scratch_bytes(n, hq, hkv, 128, ctx)
            for m in reqs[:reqs.index(n) + 1]:
                for c in ctxs[:ctxs.index(ctx) + 1]:
                    for elem in (E2M1, 1, 2):
                        d = _desc(elem, n_kv_heads=hkv)
                        got = lib.kv_op_paged_attention_batched(q, hq * 128, dtype, m, hq, C.byref(d), 0, tab, 256, lens, c, 0.1, scr, need,
                                                                out, hq * 128, None, 0)
                        assert got == CLOSED, (n, ctx, m, c, elem, got)


# ------------------------------------------------------------------ refusals of the binding
def test_binding_refuses_what_does_not_fit(kv):
    torch = pytest.importorskip("torch")
    s = synth.SHAPES["tiny"]
    cache, other = kv.PagedCache(s, 4, device="cpu", elem_bytes=0.5), kv.PagedCache(s, 5, device="cpu", elem_bytes=0.5)
    rope, bounds = kv.Rope(64), kv.BlockBounds(cache)
    rows, slots, pos = torch.zeros(3, 2, 64), torch.zeros(3, dtype=torch.int64), torch.zeros(3, dtype=torch.int32)
    q = torch.zeros(3, 4, 64)

    def append(k=rows, v=rows, pos=pos, slots=slots, q=q, out=q):
        return lambda: kv.kv_op_cache_append(rope, cache, 0, k, v, pos, slots, q=q, q_out=out)
    bad = [append(k=rows.half()), append(v=rows.bfloat16()), append(v=rows[:2]), append(k=rows[:, :1], v=rows[:, :1]), append(pos=pos.long()),
           append(pos=pos[:2]), append(pos=torch.zeros(6, dtype=torch.int32)[::2]), append(slots=slots.int()), append(slots=slots[:2]),
           append(out=None), append(q=None), append(q=q[:2], out=q[:2]), append(q=q.bfloat16(), out=q.bfloat16()), append(out=q[:, :2]),
           append(q=q[..., :32], out=q[..., :32]), append(q=torch.zeros(3, 4, 128)[..., ::2]), append()]      # the last: not on a CUDA device
    blocks, counts = torch.zeros(2, dtype=torch.int32), torch.ones(2, dtype=torch.int32)

    def bound(cache=cache, blocks=blocks, counts=counts, bounds=bounds):
        return lambda: kv.kv_op_block_bounds(cache, 0, blocks, counts, bounds)
    bad += [bound(blocks=blocks.long()), bound(blocks=blocks[None]), bound(counts=counts[:1]), bound(counts=counts.long()),
            bound(cache=other), bound(blocks=torch.zeros(4, dtype=torch.int32)[::2]), bound()]
    tab, lens = torch.zeros(2, 4, dtype=torch.int32), torch.ones(2, dtype=torch.int32)
    q, kept, kept_lens = torch.zeros(2, 4, 64), torch.zeros(2, 2, 3, dtype=torch.int32), torch.ones(2, dtype=torch.int32)

    def select(q=q, tab=tab, lens=lens, kept=kept, kept_lens=kept_lens, ctx=64):
        return lambda: kv.kv_op_select_blocks(q, bounds, 0, tab, lens, ctx, kept, kept_lens, None)
    bad += [select(q=q[0]), select(q=q[..., :32]), select(q=q.half()), select(q=q[:, ::2]), select(tab=tab.long()), select(tab=tab[:1]),
            select(tab=tab.t()), select(tab=torch.zeros(4, dtype=torch.int32).expand(2, 4)), select(lens=lens[:1]), select(lens=lens.long()),
            select(kept=kept[:1]), select(kept=kept[0]), select(kept=kept[0, 0, 0]), select(kept=kept[:, :1]), select(kept=kept.long()), select(kept=kept[..., :2]), select(kept_lens=kept_lens.long()),
            select()]

    def attend(q=q, kept=kept, lens=kept_lens, out=q, lse=None):
        return lambda: kv.kv_op_paged_attention_selected(q, cache, 0, kept, lens, out, None, lse=lse)
    bad += [attend(q=q[..., :32]), attend(out=q[:1]), attend(out=q.bfloat16()), attend(q=q[:, ::2], out=q[:, ::2]), attend(kept=kept[:, 0]), attend(kept=kept[0, 0, 0]),
            attend(kept=kept[:, :1]), attend(kept=kept.long()), attend(kept=kept.transpose(1, 2)), attend(kept=kept[:, :1].expand(2, 2, 3)),
            attend(lens=kept_lens[:1]), attend(lens=kept_lens.long()), attend(lse=torch.zeros(2, 3)), attend(lse=torch.zeros(2, 4).double()),
            attend()]
    for i, f in enumerate(bad):
        with pytest.raises(ValueError):
            f()
            pytest.fail(f"call {i} was taken")
    for call in (select(ctx=65), lambda: kv.kv_op_block_bounds(cache, 2, blocks, counts, bounds),
                 lambda: kv.kv_op_block_bounds(cache, -1, blocks, counts, bounds)):
        with pytest.raises(kv.KVError):
            call()


def test_numbers_past_32_bits_are_refused_not_cut(kv):
    torch = pytest.importorskip("torch")
    cache, big = kv.PagedCache(synth.SHAPES["tiny"], 4, device="cpu", elem_bytes=0.5), (1 << 32) + 5
    rope, bounds = kv.Rope(64), kv.BlockBounds(cache)

    def of(*shape, dtype=torch.int32):
        return torch.empty(*shape, dtype=dtype, device="meta")
    many, rows, q = of(big, 2, 64, dtype=torch.float32), of(3, 2, 64, dtype=torch.float32), of(1, 4, 64, dtype=torch.float32)
    calls = [lambda: kv.kv_op_cache_append(rope, cache, 0, many, many, of(big), of(big, dtype=torch.int64)),
             lambda: kv.kv_op_cache_append(rope, cache, 1 << 32, rows, rows, of(3), of(3, dtype=torch.int64)),
             lambda: kv.kv_op_cache_append(rope, cache, 0, rows, rows, of(3), of(3, dtype=torch.int64),
                                           q=of(3, big, 64, dtype=torch.float32), q_out=of(3, big, 64, dtype=torch.float32)),
             lambda: kv.kv_op_block_bounds(cache, 0, of(big), of(big), bounds),
             lambda: kv.kv_select_blocks_scratch_bytes(big, cache, 16),
             lambda: kv.kv_select_blocks_scratch_bytes(1, bounds, big),
             lambda: kv.kv_op_select_blocks(q, bounds, 0, of(1, big), of(1), big, of(1, 2, 4), of(1), None),
             lambda: kv.kv_op_select_blocks(q, bounds, 0, of(1, 4), of(1), 16, of(1, 2, big), of(1), None),
             lambda: kv.kv_op_select_blocks(q, bounds, 0, of(1, 4), of(1), 16, of(1, 2, 4), of(1), None, first=big),
             lambda: kv.kv_op_paged_attention_selected(q, cache, 0, of(1, 2, big), of(1), q, None),
             lambda: kv.kv_op_paged_attention_selected(q, cache, 1 << 32, of(1, 2, 4), of(1), q, None)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="32-bit"):
            call()
            pytest.fail(f"call {i} was taken")
