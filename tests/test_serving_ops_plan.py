"""How the batched attention cuts its work, as far as the scratch size shows it (no GPU needed; 148 SMs without one)."""
import pytest


@pytest.fixture(scope="module")
def lib():
    import paper_2608_16477_b200 as kv
    return kv.load()


def _records(lib, n_req, kv_heads, ctx, group=8, dim=128):
    """Bytes of the scratch that hold records: what the starts of the requests leave."""
    whole = lib.kv_paged_attention_batched_scratch_bytes(n_req, group * kv_heads, kv_heads, dim, ctx)
    return whole - -(-(n_req + 1) * 8 // 256) * 256


@pytest.mark.parametrize("kv_heads,group", [(2, 8), (1, 16), (2, 1)])
def test_heads_that_leave_half_of_a_cta_idle_keep_four_warps_each(lib, kv_heads, group):
    """A warp per KV head makes more ranges, hence records, than four do.  One or two heads (or passes over one) are not given a
    warp each, however many requests there are: the CTA's other warps would have nothing to load."""
    for ctx in (600, 4096):
        few = _records(lib, 50, kv_heads, ctx, group)      # enough keys for every range, too few requests for a warp each
        assert [_records(lib, n, kv_heads, ctx, group) for n in (100, 700, 5000)] == [few] * 3


@pytest.mark.parametrize("kv_heads", [4, 8, 16])
def test_heads_that_fill_the_ctas_take_a_warp_each_in_large_batches(lib, kv_heads):
    assert _records(lib, 8, kv_heads, 4096) < _records(lib, 700, kv_heads, 4096)


@pytest.mark.parametrize("kv_heads", [1, 2, 3, 5, 6, 8])
@pytest.mark.parametrize("n_req", [8, 100, 300, 700])
def test_scratch_grows_with_the_context(lib, kv_heads, n_req):
    sizes = [lib.kv_paged_attention_batched_scratch_bytes(n_req, 8 * kv_heads, kv_heads, 128, c)
             for c in (1, 384, 385, 511, 512, 513, 768, 769, 1024, 1025, 4096, 100000)]
    assert sizes == sorted(sizes)


FAKE = 0x7000000000


@pytest.mark.parametrize("kv_heads", [1, 2, 3, 5, 6, 7, 8])
def test_scratch_serves_fewer_requests_and_shorter_contexts(lib, kv_heads):
    """No call on a larger call's scratch is refused (the fake addresses get as far as the missing device)."""
    torch = pytest.importorskip("torch")
    if torch.cuda.is_available():
        pytest.skip("the addresses are not real")
    import ctypes as C
    from paper_2608_16477_b200.binding import CacheDesc
    page = 16 * kv_heads * 64 * 2
    desc = CacheDesc(FAKE, 2 * 16 * page, 16 * page, page, 16, 16, 1, kv_heads, 64, 2)
    q, tab, lens, scr, out = (FAKE + i * 0x1000000 for i in range(1, 6))
    ctxs, reqs = (300, 400, 512, 513, 800, 1024, 1025, 4096), (1, 7, 8, 119, 120, 198, 300, 592, 700)
    for n in reqs:
        for ctx in ctxs:
            need = lib.kv_paged_attention_batched_scratch_bytes(n, 8 * kv_heads, kv_heads, 64, ctx)
            for m in reqs[:reqs.index(n) + 1]:
                for c in ctxs[:ctxs.index(ctx) + 1]:
                    got = lib.kv_op_paged_attention_batched(q, 512 * kv_heads, 0, m, 8 * kv_heads, C.byref(desc), 0, tab, 256, lens,
                                                            c, 0.1, scr, need, out, 512 * kv_heads, None, 0)
                    assert got == -13, (n, ctx, m, c, got)


# ------------------------------------------------------------------ refusals
def test_rope_plans_that_leave_the_kernels_range_are_refused():
    """The gain is applied in fp32: one that is infinite or zero there would make every result so.  A base that overflows when it is
    scaled would turn the first pair alone."""
    import paper_2608_16477_b200 as kv
    for bad in (dict(gain=1e39), dict(gain=1e-46), dict(gain=1e-39), dict(gain=float("inf")), dict(gain=float("nan")), dict(gain=-1.0),
                dict(base=1e300, scaling="ntk", factor=1e200)):
        with pytest.raises(kv.KVError) as e:
            kv.Rope(64, **bad)
        assert e.value.status == -1, bad
    for good in (dict(gain=3e38), dict(gain=1.2e-38), dict(base=1e300, scaling="ntk", factor=2.0)):
        kv.Rope(64, **good)


@pytest.mark.parametrize("elem", [1, 2])
def test_attention_in_place_with_other_strides_is_refused(lib, elem):
    """out may be q itself with the same strides.  With others, one request's result would overwrite another's query."""
    import ctypes as C
    from paper_2608_16477_b200.binding import CacheDesc
    page = 16 * 2 * 64 * elem + (32 if elem == 1 else 0)
    desc = CacheDesc(FAKE, 2 * 16 * page, 16 * page, page, 16, 16, 1, 2, 64, elem)
    tab, lens, scr, x, other = (FAKE + i * 0x1000000 for i in range(1, 6))

    def call(n_req, out, q_stride, out_stride):
        return lib.kv_op_paged_attention_batched(x, q_stride, 0, n_req, 4, C.byref(desc), 0, tab, 256, lens, 100, 0.1, scr, 1 << 30, out,
                                                 out_stride, None, 0)
    assert call(3, x, 256, 512) == call(3, x, 512, 256) == call(2, x, 0, 256) == -1
    import torch
    if not torch.cuda.is_available():      # these go on, as far as the missing device
        assert call(3, x, 256, 256) == call(1, x, 0, 256) == call(3, other, 512, 256) == -13


def test_numbers_past_32_bits_are_refused_not_cut():
    """2^32 + 5 tokens are not 5, layer 2^32 is not layer 0 (tensors without memory: nothing of them is read)."""
    torch = pytest.importorskip("torch")
    import paper_2608_16477_b200 as kv
    import synth
    cache, big = kv.PagedCache(synth.SHAPES["tiny"], 4, device="cpu"), (1 << 32) + 5
    rope = kv.Rope(64)
    x = torch.empty(big, 2, 64, device="meta")
    rows, slots = torch.empty(3, 2, 64, device="meta"), torch.empty(3, dtype=torch.int64, device="meta")
    q, lens = torch.empty(1, 4, 64, device="meta"), torch.empty(1, dtype=torch.int32, device="meta")
    table = torch.empty(1, big, dtype=torch.int32, device="meta")
    calls = [lambda: kv.kv_op_rope(rope, x, torch.empty(big, dtype=torch.int32, device="meta"), x),
             lambda: kv.kv_op_cache_write(cache, 0, x, x, torch.empty(big, dtype=torch.int64, device="meta")),
             lambda: kv.kv_op_cache_read(cache, 0, torch.empty(big, dtype=torch.int64, device="meta"), x, x),
             lambda: kv.kv_op_cache_write(cache, 1 << 32, rows, rows, slots),
             lambda: kv.kv_op_cache_read(cache, -(1 << 32), slots, rows, rows),
             lambda: kv.kv_op_paged_attention_batched(q, cache, 1 << 32, table, lens, 16, q, None),
             lambda: kv.kv_op_paged_attention_batched(q, cache, 0, table, lens, big, q, None),
             lambda: kv.kv_paged_attention_batched_scratch_bytes(big, 4, cache, 16),
             lambda: kv.kv_paged_attention_batched_scratch_bytes(1, 4, cache, big),
             lambda: kv.Rope((1 << 32) + 64)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError, match="32-bit"):
            call()
            pytest.fail(f"call {i} was taken")
