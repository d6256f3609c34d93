"""Block bounds, the selection of blocks and attention over the selected ones on the GPU against the oracle (oracle/pages4_oracle.py).

Bounds and selections are whole numbers: equal.  Attention over a selection is the batched attention with other tables: its tolerance
(tests/test_gpu_serving_ops.py)."""
import math

import numpy as np
import pytest

from oracle import pages4_oracle as P
from oracle import serving_oracle as S
from tests.test_gpu_serving_ops import Batch, _half_step, _np, _shape

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


# ------------------------------------------------------------------ bounds
@pytest.mark.parametrize("elem", [0.5, 1, 2])
@pytest.mark.parametrize("case", [(8, 128, 16, "layer_major"), (3, 64, 7, "block_major"), (1, 128, 1, "layer_major"), (2, 64, 32, "layer_major")],
                         ids=str)
def test_bounds(kv, torch, elem, case):
    hkv, d, block, layout = case
    nb, layer = 23, 1
    rng = np.random.default_rng(2)
    cache = kv.PagedCache(_shape(hkv, d, block, 2), nb, layout=layout, elem_bytes=elem)
    cache.data.view(torch.uint8).fill_(0xFF)                     # NaN: slots behind a block's count
    counts = rng.integers(1, block + 1, nb)
    x = rng.standard_normal((nb, block, hkv, d)).astype(np.float32) * 2.0 ** rng.integers(-30, 30, (nb, 1, hkv, 1)).astype(np.float32)
    x[2] = 0.0
    x[3, :, 0] = 127.0                                           # a bound at the end of its range, and just past it
    x[4, :, 0], x[4, 0, 0, 3] = 1.0, 127.5
    x[5, :, 0] = -np.abs(x[5, :, 0])                             # one sign only
    x[6, 0, hkv - 1, 5] = math.nan
    x[7, counts[7] - 1, 0, 0] = math.inf
    x[8, 0, 0, 1] = 127.0 * 2.0 ** 60 * 1.5                      # larger than a bound covers
    x[9, :, 0] = 2.0 ** -90
    at = [(b, s) for b in range(nb) for s in range(counts[b])]
    rows = torch.from_numpy(np.stack([x[b, s] for b, s in at])).cuda()
    slots = torch.tensor([b * block + s for b, s in at], device="cuda")
    kv.kv_op_cache_write(cache, layer, rows, rows, slots)
    back, other = torch.empty_like(rows), torch.empty_like(rows)
    kv.kv_op_cache_read(cache, layer, slots, back, other)
    keys = _np(back)
    bounds = kv.BlockBounds(cache)
    bounds.codes.fill_(77)
    bounds.scales.fill_(99)
    listed = [b for b in range(nb) if b not in (20, 21)]
    blocks = torch.tensor(listed + [-1, nb, 21, 5], dtype=torch.int32, device="cuda")      # outside the pool; no rows; twice
    given = torch.tensor([int(counts[b]) for b in listed] + [3, 3, 0, int(counts[5])], dtype=torch.int32, device="cuda")
    if block == 1:
        given[0] = 1000                                          # clamped to the block size
    kv.kv_op_block_bounds(cache, layer, blocks, given, bounds)
    codes, scales = bounds.codes.cpu().numpy(), bounds.scales.cpu().numpy()
    assert (codes[0] == 77).all() and (scales[0] == 99).all()
    assert (codes[1, 20:22] == 77).all() and (scales[1, 20:22] == 99).all()
    for b in listed:
        mine = [i for i, (bb, _) in enumerate(at) if bb == b]
        for h in range(hkv):
            want, byte = P.block_bounds(keys[mine, h])
            assert scales[1, b, h] == byte, (b, h, scales[1, b, h], byte)
            assert np.array_equal(codes[1, b, h], want), (b, h)
            if byte != P.INFINITE:
                unit = 2.0 ** (int(byte) - 127)
                assert (codes[1, b, h, 0] * unit >= keys[mine, h].max(0)).all() and (codes[1, b, h, 1] * unit <= keys[mine, h].min(0)).all()


# ------------------------------------------------------------------ selection
class Chosen:
    """A Batch with bounds of its blocks and a selection."""

    def __init__(self, kv, torch, lens, hkv, group, d, block, elem, dtype, keep, first=1, last=2, seed=0, **kw):
        self.b = b = Batch(kv, torch, lens, hkv, group, d, block, elem, dtype, seed=seed, **kw)
        self.keep, self.first, self.last, self.block = keep, first, last, block
        self.bounds = kv.BlockBounds(b.cache)
        blocks, counts = [], []
        table = b.table.cpu().numpy()
        for r, n in enumerate(b.lens):
            for i in range(-(-n // block)):
                blocks.append(int(table[r, i]))
                counts.append(min(block, n - i * block))
        if blocks:
            kv.kv_op_block_bounds(b.cache, b.layer, torch.tensor(blocks, dtype=torch.int32, device="cuda"),
                                  torch.tensor(counts, dtype=torch.int32, device="cuda"), self.bounds)
        self.kept = torch.full((len(lens), hkv, keep), 12345, dtype=torch.int32, device="cuda")
        self.kept_lens = torch.full((len(lens),), 777, dtype=torch.int32, device="cuda")
        self.select_scratch = torch.full((kv.kv_select_blocks_scratch_bytes(len(lens), b.cache, b.ctx),), 0xFF, dtype=torch.uint8, device="cuda")
        need = kv.kv_paged_attention_batched_scratch_bytes(len(lens), hkv * group, b.cache, keep * block)
        self.scratch = torch.full((need,), 0xFF, dtype=torch.uint8, device="cuda")

    def select(self, kv, **kw):
        b = self.b
        kv.kv_op_select_blocks(b.q, self.bounds, b.layer, b.table, b.lens_dev, b.ctx, self.kept, self.kept_lens, self.select_scratch,
                               first=self.first, last=self.last, **kw)

    def attend(self, kv, **kw):
        b = self.b
        kv.kv_op_paged_attention_selected(b.q, b.cache, b.layer, self.kept, self.kept_lens, b.out, self.scratch, **{**dict(lse=b.lse), **kw})

    def want(self, r, h, n=None):
        b = self.b
        n = b.lens[r] if n is None else n
        q = _np(b.q)[r, h * b.group:(h + 1) * b.group]
        table = b.table[r].cpu().numpy()
        return P.select(q, self.bounds.codes[b.layer, :, h].cpu().numpy(), self.bounds.scales[b.layer, :, h].cpu().numpy(), table, n,
                        self.block, self.keep, self.first, self.last)

    def check(self, torch, lens=None):
        b = self.b
        kept, lens_got, table = self.kept.cpu().numpy(), self.kept_lens.cpu().numpy(), b.table.cpu().numpy()
        for r, n in enumerate(b.lens if lens is None else lens):
            for h in range(b.hkv):
                blocks, length = self.want(r, h, n)
                assert lens_got[r] == length, (r, lens_got[r], length)
                assert np.array_equal(kept[r, h, :len(blocks)], table[r, blocks]), (r, h)
                assert (kept[r, h, len(blocks):] == -1).all()

    def check_attention(self, torch):
        b = self.b
        q, out, lse, half = _np(b.q), _np(b.out), _np(b.lse), _half_step(torch, b.q.dtype)
        for r, n in enumerate(b.lens):
            for h in range(b.hkv):
                mine = slice(h * b.group, (h + 1) * b.group)
                blocks, length = self.want(r, h)
                rows = [p for i in blocks for p in range(i * self.block, min(n, (i + 1) * self.block))]
                assert len(rows) == length
                o, ls, size, most = S.attend(q[r, mine], b.k[r][rows, h][:, None], b.v[r][rows, h][:, None], b.d ** -0.5)
                share = most * 2.0 ** -13 + 2.0 ** -14 + (length / 16 + 64) * 2.0 ** -22
                assert (np.abs(out[r, mine] - o) <= size * share + half * np.abs(o) * 1.01).all(), (r, h)
                if n == 0:
                    assert (lse[r] == -np.inf).all()
                else:
                    assert (np.abs(lse[r, mine] - ls) <= share + 2.0 ** -23 * np.abs(ls)).all(), (r, h)


SELECT = [  # lens, kv_heads, group, dim, block, elem, dtype, keep, first, last
    ([1], 1, 1, 64, 16, 2, "float32", 1, 0, 1),
    ([0, 1, 15, 16, 17, 100, 130], 2, 4, 128, 16, 1, "bfloat16", 4, 1, 2),
    ([500, 0, 64, 65, 80, 81], 8, 8, 128, 16, 0.5, "bfloat16", 5, 1, 2),
    ([500, 300], 3, 3, 64, 7, 2, "float32", 20, 2, 3),
    ([500, 300], 5, 2, 64, 7, 0.5, "float32", 4, 0, 4),              # the last ones alone
    ([700], 1, 16, 128, 1, 1, "float32", 200, 0, 1),                 # blocks of one token, two passes over the heads
    ([5000], 2, 4, 64, 16, 2, "bfloat16", 64, 1, 2),
    ([9000, 4100, 4112, 30], 8, 4, 128, 16, 1, "float32", 100, 3, 1),
    ([3000] * 3 + [40] * 150, 2, 2, 64, 8, 0.5, "bfloat16", 33, 1, 2),
    ([2000, 1999], 4, 8, 128, 32, 0.5, "float32", 3, 1, 2),          # no place for the score to fill
]


@pytest.mark.parametrize("case", SELECT, ids=lambda c: f"{len(c[0])}x{max(c[0])}-" + "-".join(map(str, c[1:])))
def test_select_and_attend(kv, torch, case):
    lens, hkv, group, d, block, elem, dtype, keep, first, last = case
    c = Chosen(kv, torch, lens, hkv, group, d, block, elem, getattr(torch, dtype), keep, first, last)
    c.select(kv)
    c.check(torch)
    c.attend(kv)
    c.check_attention(torch)


def test_a_selection_of_everything_is_the_whole_attention(kv, torch):
    c = Chosen(kv, torch, [600, 0, 33], 2, 4, 64, 16, 0.5, torch.bfloat16, keep=38)
    c.select(kv)
    c.attend(kv)
    got, got_lse = c.b.out.clone(), c.b.lse.clone()
    c.b.run(kv)
    # the same rows, perhaps cut into other ranges: bf16 results may differ by a rounding
    assert ((got.float() - c.b.out.float()).abs() <= 2.0 ** -7 * c.b.out.float().abs() + 1e-6).all()
    assert torch.allclose(got_lse, c.b.lse, rtol=0, atol=1e-5)


def test_equal_scores_go_to_the_lowest_positions(kv, torch):
    """All blocks alike, then two kinds of them: the choice is by position among equals, whatever their number and place."""
    n, block, hkv = 300 * 16, 16, 2
    c = Chosen(kv, torch, [n], hkv, 2, 64, block, 2, torch.float32, keep=40)
    c.bounds.codes.fill_(3)
    c.bounds.scales.fill_(127)
    c.select(kv)
    table = c.b.table[0]
    want = torch.cat([table[:38], table[298:300]])
    assert torch.equal(c.kept[0, 0], want) and torch.equal(c.kept[0, 1], want)
    better = torch.tensor([5, 70, 71, 200, 296, 297], device="cuda")
    c.bounds.codes[0, table[better].long()] = torch.tensor([4, 3], dtype=torch.int8, device="cuda").view(1, 1, 2, 1)
    c.select(kv)
    c.check(torch)
    rest = [i for i in range(1, 298) if i not in better.tolist()][:31]
    want = sorted([0, 298, 299] + better.tolist() + rest)
    assert c.kept[0, 0].tolist() == table[want].tolist()
    c.b.q.zero_()                                                   # all scores zero
    c.select(kv)
    assert torch.equal(c.kept[0, 0], torch.cat([table[:38], table[298:300]]))


def test_blocks_that_no_bound_covers_are_chosen(kv, torch):
    """Infinite keys, ids outside the pool: chosen, so that their NaN shows; more of them than places: the lowest positions."""
    c = Chosen(kv, torch, [100 * 16, 90 * 16], 2, 2, 64, 16, 2, torch.float32, keep=10)
    table = c.b.table
    c.bounds.scales[0, table[0, 50].long(), 1] = 255
    table[1, 33], table[1, 44] = -1, c.b.cache.num_blocks
    c.select(kv)
    c.check(torch)
    assert int(table[0, 50]) in c.kept[0, 1].tolist() and -1 in c.kept[1, 0].tolist()
    c.attend(kv)
    assert torch.isnan(c.b.out[1]).all() and not torch.isnan(c.b.out[0]).any()
    table[1, 20:60] = -1
    c.select(kv)
    c.check(torch)
    assert c.kept[1, 0, 1:8].tolist() == [-1] * 7


def test_queries_that_are_not_finite_or_huge(kv, torch):
    """Infinities and NaN count as zero in the score; queries at both ends of fp32."""
    c = Chosen(kv, torch, [900, 800, 700, 600], 2, 4, 64, 16, 1, torch.float32, keep=9)
    c.b.q[0, 1, 3], c.b.q[0, 2, 5], c.b.q[0, 6, 7] = math.inf, -math.inf, math.nan
    c.b.q[1] *= 2.0 ** 100
    c.b.q[2] *= 2.0 ** -110
    c.b.q[3, :4] = math.nan
    c.select(kv)
    c.check(torch)


def test_lengths_outside_the_range_and_other_strides(kv, torch):
    c = Chosen(kv, torch, [500, 400, 300], 3, 2, 64, 16, 0.5, torch.bfloat16, keep=8, ctx=500)
    b = c.b
    b.lens_dev[1] = -7
    wide = torch.full((3, 10, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    wide[:, 2:8] = b.q
    tab = torch.full((3, b.table.shape[1] + 5), 10 ** 9, dtype=torch.int32, device="cuda")
    tab[:, :b.table.shape[1]] = b.table
    kv.kv_op_select_blocks(wide[:, 2:8], c.bounds, 0, tab[:, :b.table.shape[1]], b.lens_dev, 500, c.kept, c.kept_lens, c.select_scratch)
    c.check(torch, lens=[500, 0, 300])
    b.lens_dev[0] = 10 ** 7                                          # clamped to max_ctx
    c.select(kv)
    c.check(torch, lens=[500, 0, 300])
    # attention with the kept blocks inside a wider tensor, heads of a request apart
    more = torch.full((3, 4, 12), 10 ** 9, dtype=torch.int32, device="cuda")
    more[:, :3, :8] = c.kept
    outs = torch.full((3, 12, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    kv.kv_op_paged_attention_selected(wide[:, 2:8], b.cache, 0, more[:, :3, :8], c.kept_lens, outs[:, 4:10], c.scratch)
    c.attend(kv)
    assert torch.equal(outs[:, 4:10], b.out) and (outs[:, :4] == 7).all() and (outs[:, 10:] == 7).all() and (b.out[1] == 0).all()


def test_a_long_context(kv, torch):
    """Some 300,000 tokens in blocks of 16: many rounds of the choice; random bounds stand in for keys."""
    n, hkv, d, nb = 300_001, 2, 128, 20_000
    cache = kv.PagedCache(_shape(hkv, d, 16), nb, elem_bytes=0.5, fill=0)
    bounds = kv.BlockBounds(cache)
    gen = torch.Generator(device="cuda").manual_seed(3)
    top, low = (torch.randint(-127, 128, (1, nb, hkv, d), generator=gen, device="cuda") for _ in range(2))
    bounds.codes.copy_(torch.stack([torch.maximum(top, low), torch.minimum(top, low)], 3))
    bounds.scales.copy_(torch.randint(120, 123, bounds.scales.shape, generator=gen, device="cuda"))
    table = torch.randperm(nb, generator=gen, device="cuda").to(torch.int32).view(1, -1)
    q = torch.randn(1, 8, d, generator=gen, device="cuda")
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    for keep in (64, 3000, 18_000):
        kept = torch.empty(1, hkv, keep, dtype=torch.int32, device="cuda")
        kept_lens = torch.empty(1, dtype=torch.int32, device="cuda")
        scratch = torch.empty(kv.kv_select_blocks_scratch_bytes(1, bounds, n), dtype=torch.uint8, device="cuda")
        kv.kv_op_select_blocks(q, bounds, 0, table, lens, n, kept, kept_lens, scratch, first=2, last=3)
        codes, scales, t = bounds.codes[0].cpu().numpy(), bounds.scales[0].cpu().numpy(), table[0].cpu().numpy()
        for h in range(hkv):
            u = P.query_code(_np(q)[0, h * 4:h * 4 + 4])
            blocks = -(-n // 16)
            mid = np.arange(2, blocks - 3)
            score = (codes[t[mid], h].astype(np.int64).reshape(len(mid), -1) @ u).astype(np.float32) * 2.0 ** (scales[t[mid], h].astype(np.float64) - 127)
            best = mid[np.lexsort((mid, -score))[:keep - 5]]
            want = np.sort(np.concatenate([[0, 1], best, np.arange(blocks - 3, blocks)]))
            assert np.array_equal(kept[0, h].cpu().numpy(), t[want]), (keep, h)
        assert int(kept_lens) == n - (blocks - keep) * 16


@pytest.mark.parametrize("elem", [0.5, 1, 2])
def test_a_decode_step_in_a_graph(kv, torch, elem):
    """Append, bounds, select, attend captured once and replayed token after token, against the same calls made directly and, at the end,
    the oracle."""
    r, hq, hkv, d, block, keep, steps = 3, 8, 2, 64, 16, 6, 30
    gen = torch.Generator(device="cuda").manual_seed(5)
    rope = kv.Rope(d, base=1e4)
    start = [100, 37, 200]
    ctx, nb = 256, 50
    caches = [kv.PagedCache(_shape(hkv, d, block), nb, elem_bytes=elem, fill=0) for _ in range(2)]
    bounds = [kv.BlockBounds(c) for c in caches]
    table = torch.randperm(nb, generator=gen, device="cuda")[:48].to(torch.int32).view(3, 16)
    k_all, v_all = (torch.randn(r, 256, hkv, d, generator=gen, device="cuda").bfloat16() for _ in range(2))
    for i, n in enumerate(start):                # the prefix of each request, its keys turned on the way
        at = torch.arange(n, device="cuda")
        slots = table[i].long()[at // block] * block + at % block
        for c, bd in zip(caches, bounds):
            kv.kv_op_cache_append(rope, c, 0, k_all[i, :n], v_all[i, :n], at.to(torch.int32), slots)
            blocks = table[i, :-(-n // block)].contiguous()
            counts = (n - torch.arange(len(blocks), device="cuda") * block).clamp_max(block).to(torch.int32)
            kv.kv_op_block_bounds(c, 0, blocks, counts, bd)
    q_in = torch.zeros(r, hq, d, dtype=torch.bfloat16, device="cuda")
    k, v = (torch.zeros(r, hkv, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    pos, lens, counts, blocks = (torch.zeros(r, dtype=torch.int32, device="cuda") for _ in range(4))
    slots = torch.zeros(r, dtype=torch.int64, device="cuda")
    q, out, lse = torch.empty_like(q_in), torch.empty_like(q_in), torch.empty(r, hq, device="cuda")
    kept, kept_lens = torch.empty(r, hkv, keep, dtype=torch.int32, device="cuda"), torch.empty(r, dtype=torch.int32, device="cuda")
    s1 = torch.empty(kv.kv_select_blocks_scratch_bytes(r, caches[0], ctx), dtype=torch.uint8, device="cuda")
    s2 = torch.empty(kv.kv_paged_attention_batched_scratch_bytes(r, hq, caches[0], keep * block), dtype=torch.uint8, device="cuda")

    def step(i):
        kv.kv_op_cache_append(rope, caches[i], 0, k, v, pos, slots, q=q_in, q_out=q)
        kv.kv_op_block_bounds(caches[i], 0, blocks, counts, bounds[i])
        kv.kv_op_select_blocks(q, bounds[i], 0, table, lens, ctx, kept, kept_lens, s1)
        kv.kv_op_paged_attention_selected(q, caches[i], 0, kept, kept_lens, out, s2, lse=lse)

    def lists(s):
        p = torch.tensor([n + s for n in start], dtype=torch.int32)
        pos.copy_(p)
        lens.copy_(p + 1)
        counts.copy_(p % block + 1)
        blocks.copy_(table.gather(1, (pos // block).long()[:, None])[:, 0])
        slots.copy_(blocks.long() * block + pos % block)
        for i, n in enumerate(start):
            k[i], v[i] = k_all[i, n + s], v_all[i, n + s]
        q_in.copy_(torch.randn(q_in.shape, generator=gen, device="cuda") * 0.5)
    lists(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(1)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(0)
    for s in range(steps):
        lists(s)
        out.fill_(7)
        graph.replay()
        got = out.clone(), lse.clone(), kept.clone(), kept_lens.clone()
        step(1)
        for a, b in zip(got, (out, lse, kept, kept_lens)):
            assert torch.equal(a, b), s
    assert torch.equal(caches[0].data, caches[1].data) and torch.equal(bounds[0].codes, bounds[1].codes)
    # the last step against the oracle, from the cache's contents
    for i, n in enumerate(int(x) for x in lens):
        at = torch.arange(n, device="cuda")
        slots_i = table[i].long()[at // block] * block + at % block
        ks, vs = (torch.empty(n, hkv, d, device="cuda") for _ in range(2))
        kv.kv_op_cache_read(caches[0], 0, slots_i, ks, vs)
        ks, vs = _np(ks), _np(vs)
        for h in range(hkv):
            mine = slice(h * 4, h * 4 + 4)
            codes, scales = bounds[0].codes[0, :, h].cpu().numpy().copy(), bounds[0].scales[0, :, h].cpu().numpy().copy()
            ids = table[i].cpu().numpy()
            for b in range(-(-n // block)):
                codes_b, byte = P.block_bounds(ks[b * block:(b + 1) * block, h])
                assert np.array_equal(codes[ids[b]], codes_b) and scales[ids[b]] == byte
            chosen, length = P.select(_np(q)[i, mine], codes, scales, ids, n, block, keep, 1, 2)
            assert kept[i, h, :len(chosen)].tolist() == ids[chosen].tolist() and int(kept_lens[i]) == length
            rows = [p for b in chosen for p in range(b * block, min(n, (b + 1) * block))]
            o, ls, size, most = S.attend(_np(q)[i, mine], ks[rows, h][:, None], vs[rows, h][:, None], d ** -0.5)
            share = most * 2.0 ** -13 + 2.0 ** -14 + (length / 16 + 64) * 2.0 ** -22
            assert (np.abs(_np(out)[i, mine] - o) <= size * share + 2.0 ** -8 * np.abs(o) * 1.01).all()


def test_two_selections_at_once(kv, torch):
    """Two batches on two streams at the same time, each with scratch of its own, over and over."""
    a = Chosen(kv, torch, [3000, 90, 700], 8, 8, 128, 16, 0.5, torch.bfloat16, keep=20)
    b = Chosen(kv, torch, [2500, 1, 0, 1800], 8, 4, 128, 16, 2, torch.float32, keep=12, seed=2)
    for x in (a, b):
        x.select(kv)
        x.attend(kv)
    torch.cuda.synchronize()
    want = [(x.kept.clone(), x.b.out.clone()) for x in (a, b)]
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    for _ in range(30):
        for x, s in zip((a, b), streams):
            x.select(kv, stream=s)
            x.attend(kv, stream=s)
    torch.cuda.synchronize()
    for x, (kept, out) in zip((a, b), want):
        assert torch.equal(x.kept, kept) and torch.equal(x.b.out, out)


@pytest.mark.parametrize("kind,ctx", [(kind, ctx) for kind in ("apart", "equal", "one far", "few values", "infinite")
                                      for ctx in (15 * 16 + 1, 700 * 16, 2051 * 16, 2600 * 16 + 3)] +
                         [(kind, blocks * 16) for kind in ("apart", "few values") for blocks in (16384, 16385)])
def test_scores_of_every_distribution(kv, torch, kind, ctx):
    """Scores that spread, that are one value, that lie close together but for one, that take few values, with many that no bound covers:
    each asks for another way to the block of the last rank.  Bounds are given, not formed: any bytes are bounds."""
    heads, d, block, keep = 2, 64, 16, 12
    n = -(-ctx // block)
    rng = np.random.default_rng(n)
    codes = rng.integers(-127, 128, (n, heads, 2, d)).astype(np.int8)
    scales = np.full((n, heads), 127 - 7, np.uint8)
    if kind == "equal":
        codes[:] = codes[:1]
    elif kind == "one far":
        codes[:] = codes[:1] // 8
        codes[:, :, 0, 0] = rng.integers(-3, 4, (n, heads))
        scales[:] = 40
        scales[n // 2] = 140
    elif kind == "few values":
        codes[:] = codes[rng.integers(0, 5, n)]
    elif kind == "infinite":
        scales[rng.integers(0, n, n // 3)] = 255
    cache = kv.PagedCache(_shape(heads, d, block, 1), n, elem_bytes=2)
    bounds = kv.BlockBounds(cache)
    bounds.codes[0].copy_(torch.from_numpy(codes.reshape(bounds.codes[0].shape)))
    bounds.scales[0].copy_(torch.from_numpy(scales.reshape(bounds.scales[0].shape)))
    q = torch.from_numpy(rng.standard_normal((1, 2 * heads, d)).astype(np.float32)).cuda()
    table = torch.from_numpy(rng.permutation(n).astype(np.int32)[None]).cuda()
    lens = torch.tensor([ctx], dtype=torch.int32, device="cuda")
    kept = torch.empty(1, heads, keep, dtype=torch.int32, device="cuda")
    kept_lens = torch.empty(1, dtype=torch.int32, device="cuda")
    scratch = torch.empty(max(kv.kv_select_blocks_scratch_bytes(1, cache, ctx), 16), dtype=torch.uint8, device="cuda")
    kv.kv_op_select_blocks(q, bounds, 0, table, lens, ctx, kept, kept_lens, scratch)
    torch.cuda.synchronize()
    for h in range(heads):
        at = table[0].cpu().numpy()
        blocks, length = P.select(_np(q)[0, 2 * h:2 * h + 2], codes[:, h], scales[:, h], at, ctx, block, keep, 1, 2)
        assert kept_lens.tolist() == [length]
        assert np.array_equal(kept[0, h].cpu().numpy(), at[blocks])
