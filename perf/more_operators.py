"""Cases, plain forms and exact values of the operators around a KV cache held in four bits.

  append  keys and values of new tokens into pages, the rotary position applied on the way (queries turned beside them)
  attend  attention of one new token per request over e2m1 pages
  bounds  per block and KV head, the range of the cached keys in every dimension, in 8 bits
  sparse  the blocks that those bounds rank highest for a query, and attention over them alone

e2m1 pages: for every KV head a record [slot][dim / 2] of codes (two to a byte, the even dim low), [slot][dim / 16] e4m3
scales of 16 dims, [slot] scale bytes 2^(byte - 127) of the row, padded to 16 bytes.  bf16 and e4m3 pages: [slot][kv_head][dim]
values; e4m3 pages end with scale bytes [kv_head][slot], padded to 16.  Where `own` is true, `run` calls the library's operators
instead of the plain forms.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
MIN_EXP, MAX_EXP = -110, 119          # exponents that the scale of a row may take
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
FIRST, LAST = 1, 2                    # blocks at either end of a context that are always attended to


def listed():
    return [
        # the resumed decode step of one request of the 32B shape (64 query and 8 KV heads of 128), bf16 pages: latency
        dict(name="append-1", op="append", tokens=1, q_heads=64, kv_heads=8, dim=128, rotary=128, layout="half", block=16,
             bits=16, type="bf16", far=4096),
        # 64 resident requests each append one token to a 4-bit cache
        dict(name="append-64", op="append", tokens=64, q_heads=64, kv_heads=8, dim=128, rotary=128, layout="half", block=16,
             bits=4, type="bf16", far=32768),
        # the chunks of a 16k prefix of the 8B shape into a 4-bit cache
        dict(name="append-16384", op="append", tokens=16384, q_heads=32, kv_heads=8, dim=128, rotary=128, layout="half",
             block=16, bits=4, type="bf16", far=32768),
        # one short request of the tiny shape: latency
        dict(name="attend-1x161", op="attend", requests=1, ctx=161, q_heads=4, kv_heads=2, dim=64, block=16, bits=4,
             type="f32", lens=1),
        # one long request of the 32B shape: the context has to be split
        dict(name="attend-1x18433", op="attend", requests=1, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16, bits=4,
             type="bf16", lens=2),
        # many short ragged requests of the 8B shape, fp32 queries
        dict(name="attend-128x577", op="attend", requests=128, ctx=577, q_heads=32, kv_heads=8, dim=128, block=16, bits=4,
             type="f32", lens=4),
        # a full server: 32 ragged requests of the 32B shape
        dict(name="attend-32x18433", op="attend", requests=32, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16, bits=4,
             type="bf16", lens=5),
        # after a decode step: the last blocks of 64 requests
        dict(name="bounds-64", op="bounds", blocks=64, kv_heads=8, dim=128, block=16, bits=4),
        # after a prefill: every block of four 16k prefixes
        dict(name="bounds-4096", op="bounds", blocks=4096, kv_heads=8, dim=128, block=16, bits=16),
        # one long request of the 32B shape over an 8-bit cache, 64 of 1,153 blocks
        dict(name="sparse-1x18433", op="sparse", requests=1, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16, bits=8,
             type="bf16", keep=64, lens=2),
        # ragged requests of the 8B shape with fp32 queries over bf16 pages, some of them shorter than what is kept
        dict(name="sparse-16x8192", op="sparse", requests=16, ctx=8192, q_heads=32, kv_heads=8, dim=128, block=16, bits=16,
             type="f32", keep=48, lens=3),
        # a full server over a 4-bit cache
        dict(name="sparse-32x18433", op="sparse", requests=32, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16, bits=4,
             type="bf16", keep=64, lens=5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["append", "append", "attend", "attend", "bounds", "sparse", "sparse"])
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["bf16", "f32"])
    block = rng.choice([8, 16, 32])
    if op == "append":
        return dict(op=op, tokens=_log(rng, 1, 12000), q_heads=kv_heads * rng.choice([0, 1, 4, 8]), kv_heads=kv_heads, dim=dim,
                    rotary=rng.choice([dim, dim // 2, dim - 2 * rng.randint(0, dim // 4)]),
                    layout=rng.choice(["half", "interleaved"]), block=block, bits=rng.choice([4, 4, 8, 16]), type=kind,
                    far=_log(rng, 16, 1000000))
    if op == "bounds":
        return dict(op=op, blocks=_log(rng, 1, 4000), kv_heads=kv_heads, dim=dim, block=block, bits=rng.choice([4, 8, 16]))
    requests = _log(rng, 1, 128)
    case = dict(op=op, requests=requests, ctx=_log(rng, 1, max(1, min(16384, 250000 // requests))),
                q_heads=kv_heads * rng.choice([1, 2, 4, 8]), kv_heads=kv_heads, dim=dim, block=block, bits=4, type=kind,
                lens=rng.randrange(1 << 20))
    if op == "sparse":
        case.update(bits=rng.choice([4, 8, 16]), keep=_log(rng, FIRST + LAST, 128))
    return case


# ---------------------------------------------------------------- what a program has in hand before the call

def _page_bytes(case):
    rows = case["block"] * case["kv_heads"]
    if case["bits"] == 4:
        return case["kv_heads"] * (-(-case["block"] * (case["dim"] // 2 + case["dim"] // 16 + 1) // 16) * 16)
    return rows * case["dim"] * 2 if case["bits"] == 16 else rows * case["dim"] + -(-rows // 16) * 16


def _lens(case):
    """Context lengths of the batch: the longest first, the others spread over the range, one padded row of none."""
    rng = random.Random(case["lens"])
    lens = [case["ctx"]] + [rng.randint(1, case["ctx"]) for _ in range(case["requests"] - 1)]
    if case["requests"] >= 4:
        lens[2] = 0
    return lens


def _rows(gen, shape):
    """Rows as a projection leaves them: normal values, rows of different sizes, a few large channels."""
    x = torch.randn(shape, generator=gen, device=DEVICE)
    x *= torch.exp2(torch.randint(-3, 3, shape[:-1], generator=gen, device=DEVICE).float()).unsqueeze(-1)
    x[..., :: 37] *= 8
    return x


E4M3 = torch.arange(1, 127, dtype=torch.uint8).view(torch.float8_e4m3fn).float()       # the positive ones, ascending
E2M1 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
MIDS = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])


def _power(most, part, top):
    """The least integer e with most <= part * 2^top * 2^e, 0.5 <= part < 1."""
    m, power = torch.frexp(most)
    power = (power - top + (m > part).int()).clamp(MIN_EXP, MAX_EXP)
    return torch.where(most > 0, power, torch.full_like(power, MIN_EXP))


def _quantised8(x):
    """(codes, scale bytes) of rows of e4m3 pages."""
    fine = torch.isfinite(x)
    power = _power(torch.where(fine, x.abs(), torch.zeros_like(x)).amax(-1), 0.875, 9)             # 448
    scaled = (x * torch.exp2(-power.float()).unsqueeze(-1)).clamp(-448.0, 448.0)
    scaled = torch.where(fine, scaled, torch.full_like(scaled, math.nan))
    return scaled.to(torch.float8_e4m3fn), (power + 127).to(torch.uint8)


def _quantised4(x):
    """(codes 0 to 15, scale codes of 16 dims, scale bytes) of rows of e2m1 pages: the row's scale is the least power of two with
    max |x| <= 6 * 448 * 2^e, a group's the least e4m3 number with max |x| <= 6 * s * 2^e; halves between two codes go up."""
    fine = torch.isfinite(x)
    size = torch.where(fine, x.abs(), torch.zeros_like(x))
    power = _power(size.amax(-1), 0.65625, 12).clamp_max(116)                 # 2688; what is stored stays in fp32's range
    size = (size * torch.exp2(-power.float()).unsqueeze(-1)).unflatten(-1, (-1, 16))
    scale = (1 + torch.searchsorted(6.0 * E4M3.to(x.device), size.amax(-1).contiguous())).clamp_max(126)
    border = E4M3.to(x.device)[scale - 1].unsqueeze(-1)
    mids = MIDS.to(x.device)
    codes = (size >= mids[0] * border).int()
    codes += (size >= mids[1] * border).int() + (size >= mids[2] * border).int() + (size >= mids[3] * border).int()
    codes += (size >= mids[4] * border).int() + (size >= mids[5] * border).int() + (size >= mids[6] * border).int()
    codes += 8 * torch.signbit(x).int().unflatten(-1, (-1, 16))
    whole = fine.unflatten(-1, (-1, 16)).all(-1)
    codes = torch.where(whole.unsqueeze(-1), codes, torch.zeros_like(codes)).flatten(-2)
    scale = torch.where(whole, scale, torch.full_like(scale, 127))                                  # a NaN
    return codes.to(torch.uint8), scale.to(torch.uint8), (power + 127).to(torch.uint8)


def _views(case, pages):
    """Views of a tensor of pages [..., page bytes]: values of bf16 pages; codes and scale bytes [..., kv_heads, block] of e4m3
    pages; packed codes [..., kv_heads, block, dim / 2], scales of 16 dims and scale bytes [..., kv_heads, block] of e2m1 pages."""
    n, heads, block, dim = case["block"] * case["kv_heads"], case["kv_heads"], case["block"], case["dim"]
    if case["bits"] == 16:
        return {"values": pages.view(torch.bfloat16).unflatten(-1, (block, heads, dim))}
    if case["bits"] == 8:
        return {"codes": pages[..., : n * dim].view(torch.float8_e4m3fn).unflatten(-1, (block, heads, dim)),
                "rows": pages[..., n * dim: n * dim + n].unflatten(-1, (heads, block))}
    records = pages.unflatten(-1, (heads, -1))
    at, end = block * dim // 2, block * (dim // 2 + dim // 16)
    return {"codes": records[..., :at].unflatten(-1, (block, dim // 2)),
            "groups": records[..., at:end].unflatten(-1, (block, dim // 16)), "rows": records[..., end: end + block]}


def _put(case, views, rows, where):
    """Rows [..., kv_heads, dim] (fp32) into the views of pages [K, V][blocks]: where(view of one slot per row, values)."""
    if case["bits"] == 16:
        where(views["values"], rows.to(torch.bfloat16), True)
    elif case["bits"] == 8:
        codes, powers = _quantised8(rows)
        where(views["codes"].view(torch.uint8), codes.view(torch.uint8), True)
        where(views["rows"], powers, False)
    else:
        codes, scales, powers = _quantised4(rows)
        where(views["codes"], codes[..., 0::2] | (codes[..., 1::2] << 4), False)
        where(views["groups"], scales, False)
        where(views["rows"], powers, False)


def _filled(case, gen, blocks):
    """A pool [1 layer][K, V][blocks][page bytes] of written pages."""
    pages = torch.zeros(1, 2, blocks, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
    rows = _rows(gen, (2, blocks, case["block"], case["kv_heads"], case["dim"]))

    def where(view, new, slot_first):
        view[0] = new if slot_first else new.transpose(2, 3)
    _put(case, _views(case, pages), rows, where)
    return pages


def _decoded(case, pages):
    """Pages [..., page bytes] as fp32 rows [..., block, kv_heads, dim]."""
    views = _views(case, pages)
    if case["bits"] == 16:
        return views["values"].float()
    power = torch.exp2(views["rows"].float() - 127.0).transpose(-1, -2).unsqueeze(-1)
    if case["bits"] == 8:
        return views["codes"].float() * power
    packed = views["codes"]
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).int()
    values = torch.cat([E2M1, -E2M1]).to(pages.device)[codes].unflatten(-1, (-1, 16))
    values = values * views["groups"].contiguous().view(torch.float8_e4m3fn).float().unsqueeze(-1)
    return values.flatten(-2).transpose(-2, -3) * power


def _bounds_of(case, keys):
    """(codes int8 [..., kv_heads, 2, dim], scale bytes [..., kv_heads]) of rows [..., block, kv_heads, dim]: the largest value
    of each dim rounded up and the smallest rounded down, times the least power of two that leaves them in 7 bits and a sign."""
    most, least = keys.amax(-3), keys.amin(-3)
    size = torch.maximum(most.abs(), least.abs()).amax(-1)
    m, power = torch.frexp(size)
    power = (power - 7 + (m > 0.9921875).int()).clamp_min(-60)                                      # 127
    power = torch.where(size > 0, power, torch.full_like(power, -60))
    inv = torch.exp2(-power.float()).unsqueeze(-1)
    codes = torch.stack([torch.ceil(most * inv), torch.floor(least * inv)], -2)
    return codes.to(torch.int8), (power + 127).to(torch.uint8)


def _theta(case):
    """Frequencies of the rotated pairs, in 64 bits."""
    half = case["rotary"] // 2
    return 1.0e6 ** (-np.arange(half, dtype=np.float64) / half)


def _prepare_append(case, gen, state):
    blocks = -(-case["tokens"] // case["block"]) + 3
    table = torch.randperm(blocks, generator=gen, device=DEVICE)
    at = torch.arange(case["tokens"], device=DEVICE)
    state["slots"] = table[at // case["block"]] * case["block"] + at % case["block"]
    state["pages"] = torch.zeros(1, 2, blocks, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
    heads = case["q_heads"] + 2 * case["kv_heads"]
    qkv = _rows(gen, (case["tokens"], heads, case["dim"])).to(TYPES[case["type"]])
    state["q"], state["k"] = qkv[:, : case["q_heads"]], qkv[:, case["q_heads"]: case["q_heads"] + case["kv_heads"]]
    state["v"] = qkv[:, case["q_heads"] + case["kv_heads"]:]
    state["q_out"] = torch.empty(case["tokens"], case["q_heads"], case["dim"], dtype=TYPES[case["type"]], device=DEVICE)
    first = torch.randint(0, max(1, case["far"] - case["tokens"]), (1,), generator=gen, device=DEVICE)
    state["positions"] = (first + at).to(torch.int32)
    state["theta"] = torch.from_numpy(_theta(case)).to(DEVICE)


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    state = {"case": case, "own": None}
    if case["op"] == "append":
        _prepare_append(case, gen, state)
        return state
    if case["op"] == "bounds":
        pool = case["blocks"] + 5
        state["pages"] = _filled(case, gen, pool)
        state["blocks"] = torch.randperm(pool, generator=gen, device=DEVICE)[: case["blocks"]].to(torch.int32)
        counts = torch.full((case["blocks"],), case["block"], dtype=torch.int32, device=DEVICE)
        some = torch.randint(1, case["block"] + 1, (case["blocks"],), generator=gen, device=DEVICE).to(torch.int32)
        state["counts"] = torch.where(torch.arange(case["blocks"], device=DEVICE) % 4 == 3, some, counts)
        state["codes"] = torch.zeros(1, pool, case["kv_heads"], 2, case["dim"], dtype=torch.int8, device=DEVICE)
        state["scales"] = torch.zeros(1, pool, case["kv_heads"], dtype=torch.uint8, device=DEVICE)
        return state
    lens = _lens(case)
    need = [-(-n // case["block"]) for n in lens]
    blocks = sum(need) + 5
    table = torch.full((case["requests"], max(need)), -1, dtype=torch.int32)
    order = torch.randperm(blocks, generator=torch.Generator().manual_seed(int(seed))).to(torch.int32)
    taken = 0
    for r, n in enumerate(need):
        table[r, :n] = order[taken: taken + n]
        taken += n
    state["pages"] = _filled(case, gen, blocks)
    state["table"], state["lens"] = table.to(DEVICE), torch.tensor(lens, dtype=torch.int32, device=DEVICE)
    q = 0.25 * torch.randn(case["requests"], case["q_heads"], case["dim"], generator=gen, device=DEVICE)
    state["q"] = q.to(TYPES[case["type"]])
    state["out"] = torch.empty_like(state["q"])
    state["lse"] = torch.empty(case["requests"], case["q_heads"], device=DEVICE)
    if case["op"] == "sparse":
        codes, scales = _bounds_of(case, _decoded(case, state["pages"][0, 0]))
        state["codes"], state["scales"] = codes.unsqueeze(0), scales.unsqueeze(0)
        state["kept"] = torch.empty(case["requests"], case["kv_heads"], case["keep"], dtype=torch.int32, device=DEVICE)
        state["kept_lens"] = torch.empty(case["requests"], dtype=torch.int32, device=DEVICE)
    return state


# ---------------------------------------------------------------- one pass

def _values(case, views):
    """The pages' contents, as the values that they stand for."""
    if case["bits"] == 16:
        return {"values": views["values"]}
    got = {"rows": views["rows"].view(torch.float8_e8m0fnu)}
    if case["bits"] == 8:
        return {"codes": views["codes"], **got}
    packed = views["codes"]
    codes = torch.stack([packed & 15, packed >> 4], -1).flatten(-2).int()
    table = torch.cat([E2M1, -E2M1]).to(torch.float8_e4m3fn).to(packed.device)
    return {"codes": table.view(torch.uint8)[codes].view(torch.float8_e4m3fn),
            "groups": views["groups"].contiguous().view(torch.float8_e4m3fn), **got}


def _turned(case, x, cos, sin):
    half = case["rotary"] // 2
    part = x[..., : case["rotary"]].float()
    if case["layout"] == "half":
        a, b = part[..., :half], part[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., case["rotary"]:]], -1)


def _plain_append(s):
    case = s["case"]
    angle = s["positions"].double().unsqueeze(-1) * s["theta"]
    cos, sin = torch.cos(angle).float().unsqueeze(1), torch.sin(angle).float().unsqueeze(1)
    both = torch.stack([_turned(case, s["k"], cos, sin), s["v"]]).float()
    at, slot = s["slots"] // case["block"], s["slots"] % case["block"]
    views = _views(case, s["pages"][0])

    def where(view, new, slot_first):
        if slot_first:
            view[:, at, slot] = new
        else:
            view[:, at, :, slot] = new.transpose(0, 1)
    _put(case, views, both, where)
    return {"q": _turned(case, s["q"], cos, sin), **_values(case, views)}


def _attention(case, q, k, v, lens):
    """(out, lse) of queries [R, Hq, d] over rows [R, Hkv, n, d]."""
    q = q.float().unflatten(1, (case["kv_heads"], -1)) / math.sqrt(case["dim"])
    score = q @ k.transpose(-1, -2)
    seen = torch.arange(k.shape[2], device=DEVICE) < lens.unsqueeze(-1)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    weight = torch.exp(score - most)
    total = weight.sum(-1, keepdim=True)
    none = (lens == 0).view(-1, 1, 1)
    out = ((weight @ v) / total).flatten(1, 2).masked_fill(none, 0.0)
    lse = (most + torch.log(total)).flatten(1).masked_fill(none[..., 0], -math.inf)
    return out, lse


def _plain_attend(s):
    case, at = s["case"], s["table"].clamp_min(0).long()
    k = _decoded(case, s["pages"][0, 0][at]).flatten(1, 2).permute(0, 2, 1, 3)      # [R, Hkv, n, d]
    v = _decoded(case, s["pages"][0, 1][at]).flatten(1, 2).permute(0, 2, 1, 3)
    out, lse = _attention(case, s["q"], k, v, s["lens"])
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _plain_bounds(s):
    case = s["case"]
    keys = _decoded(case, s["pages"][0, 0][s["blocks"].long()])
    slot = torch.arange(case["block"], device=DEVICE)
    there = torch.minimum(slot, s["counts"].unsqueeze(-1) - 1).long()              # rows behind the last: the last again
    keys = keys.gather(1, there.view(*there.shape, 1, 1).expand_as(keys))
    codes, scales = _bounds_of(case, keys)
    s["codes"][0, s["blocks"].long()] = codes
    s["scales"][0, s["blocks"].long()] = scales
    return {"codes": s["codes"], "scales": s["scales"]}


def _plain_select(s):
    """The physical ids of the blocks that are attended to, in the order of their positions, per request and KV head; the length
    of the context that they make.  The score is a whole number times a power of two: it does not depend on the order of a sum."""
    case = s["case"]
    q = s["q"].double().unflatten(1, (case["kv_heads"], -1))
    u = torch.cat([q.clamp_min(0).sum(2), q.clamp_max(0).sum(2)], -1)                       # [R, Hkv, 2 d]
    m, power = torch.frexp(u.abs().amax(-1, keepdim=True))
    power = (power - 15 + (m > 32767 / 32768).int()).clamp_min(-100)
    u = torch.round(u * torch.exp2(-power.double()))
    n = (s["lens"] + case["block"] - 1) // case["block"]
    at = s["table"].clamp_min(0).long()
    codes = s["codes"][0][at].flatten(-2).permute(0, 2, 1, 3).double()                      # [R, Hkv, blocks, 2 d]
    sums = (codes @ u.unsqueeze(-1)).squeeze(-1).float()
    score = (sums * torch.exp2(s["scales"][0][at].float() - 127.0).transpose(1, 2)).double()
    index = torch.arange(at.shape[1], device=DEVICE)
    ends = (index < FIRST) | (index >= n.unsqueeze(-1) - LAST)
    score = score.masked_fill(ends.unsqueeze(1), 1e300).masked_fill((index >= n.unsqueeze(-1)).unsqueeze(1), -1e300)
    ranked = torch.sort(score, dim=-1, descending=True, stable=True).indices[..., : case["keep"]]
    ranked = torch.nn.functional.pad(ranked, (0, case["keep"] - ranked.shape[-1]))
    kept = torch.minimum(n, torch.full_like(n, case["keep"])).unsqueeze(-1)
    there = torch.arange(case["keep"], device=DEVICE) < kept
    ranked = ranked.masked_fill(~there.unsqueeze(1), 1 << 40).sort(-1).values
    blocks = s["table"].unsqueeze(1).expand(-1, case["kv_heads"], -1).gather(2, ranked.masked_fill(~there.unsqueeze(1), 0))
    blocks = blocks.masked_fill(~there.unsqueeze(1), -1)
    return blocks, (s["lens"] - (n - kept.squeeze(-1)) * case["block"]).to(torch.int32)


def _plain_sparse(s):
    case = s["case"]
    kept, lens = _plain_select(s)
    at, head = kept.clamp_min(0).long(), torch.arange(case["kv_heads"], device=DEVICE).view(1, -1, 1)
    rows = _decoded(case, s["pages"][0]).permute(0, 1, 3, 2, 4)                             # [2, blocks, Hkv, block, d]
    k, v = rows[0][at, head].flatten(2, 3), rows[1][at, head].flatten(2, 3)                 # [R, Hkv, n, d]
    out, lse = _attention(case, s["q"], k, v, lens)
    return {"out": out.to(s["q"].dtype), "lse": lse, "kept": kept, "lens": lens}


def _cache(s):
    """The library's cache over the state's pages."""
    import paper_2608_16477_b200 as kv
    from synth.configs import ModelShape
    case = s["case"]
    shape = ModelShape("cache", 1, case["dim"], case["kv_heads"], case["kv_heads"], case["dim"], 8, 1,
                       block_size=case["block"])
    return kv.PagedCache(shape, s["pages"].shape[2], elem_bytes={16: 2, 8: 1, 4: 0.5}[case["bits"]], data=s["pages"])


def _handles(s):
    """What a program keeps beside its inputs: the cache's descriptor, the rotary plan, the bounds, scratch."""
    import paper_2608_16477_b200 as kv
    case = s["case"]
    cache = _cache(s)
    if case["op"] == "append":
        return cache, kv.Rope(case["rotary"], layout=case["layout"], base=1.0e6)
    if case["op"] == "bounds":
        return cache, kv.BlockBounds(cache, codes=s["codes"], scales=s["scales"])
    tokens = case["ctx"] if case["op"] == "attend" else case["keep"] * case["block"]
    need = kv.kv_paged_attention_batched_scratch_bytes(case["requests"], case["q_heads"], cache, tokens)
    scratch = torch.empty(need, dtype=torch.uint8, device=DEVICE)
    if case["op"] == "attend":
        return cache, scratch
    need = kv.kv_select_blocks_scratch_bytes(case["requests"], cache, case["ctx"])
    return cache, scratch, kv.BlockBounds(cache, codes=s["codes"], scales=s["scales"]), \
        torch.empty(need, dtype=torch.uint8, device=DEVICE)


def _own(s):
    import paper_2608_16477_b200 as kv
    case = s["case"]
    if s["own"] is None:
        s["own"] = _handles(s)
    if case["op"] == "append":
        cache, rope = s["own"]
        if case["q_heads"]:
            kv.kv_op_cache_append(rope, cache, 0, s["k"], s["v"], s["positions"], s["slots"], q=s["q"], q_out=s["q_out"])
        else:
            kv.kv_op_cache_append(rope, cache, 0, s["k"], s["v"], s["positions"], s["slots"])
        return {"q": s["q_out"], **_values(case, _views(case, s["pages"][0]))}
    if case["op"] == "bounds":
        cache, bounds = s["own"]
        kv.kv_op_block_bounds(cache, 0, s["blocks"], s["counts"], bounds)
        return {"codes": s["codes"], "scales": s["scales"]}
    if case["op"] == "attend":
        cache, scratch = s["own"]
        kv.kv_op_paged_attention_batched(s["q"], cache, 0, s["table"], s["lens"], case["ctx"], s["out"], scratch,
                                         lse=s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    cache, scratch, bounds, select = s["own"]
    kv.kv_op_select_blocks(s["q"], bounds, 0, s["table"], s["lens"], case["ctx"], s["kept"], s["kept_lens"], select,
                           first=FIRST, last=LAST)
    kv.kv_op_paged_attention_selected(s["q"], cache, 0, s["kept"], s["kept_lens"], s["out"], scratch, lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"], "kept": s["kept"], "lens": s["kept_lens"]}


def run(state):
    if own:
        return _own(state)
    return {"append": _plain_append, "attend": _plain_attend, "bounds": _plain_bounds,
            "sparse": _plain_sparse}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def _row_bytes(case):
    """A token's K or V of all heads in a page."""
    dim = case["dim"]
    return case["kv_heads"] * {16: 2 * dim, 8: dim + 1, 4: dim // 2 + dim // 16 + 1}[case["bits"]]


def work(case):
    size = 2 if case.get("type") == "bf16" else 4
    row = _row_bytes(case)
    if case["op"] == "append":
        rows, dim = case["tokens"] * (2 * case["q_heads"] + 2 * case["kv_heads"]), case["dim"]     # q in and out, k and v in
        turned = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["rotary"]
        return {"bytes": rows * dim * size + 2 * case["tokens"] * row + 12 * case["tokens"],
                "flops": 3 * turned + 4 * case["tokens"] * case["kv_heads"] * dim}
    entry = case["kv_heads"] * (2 * case["dim"] + 1)                                               # a block's bounds
    if case["op"] == "bounds":
        return {"bytes": case["blocks"] * (case["block"] * row + entry + 8),
                "flops": 2 * case["blocks"] * case["block"] * case["kv_heads"] * case["dim"]}
    lens = _lens(case)
    blocks = [-(-n // case["block"]) for n in lens]
    values = case["requests"] * case["q_heads"] * case["dim"]
    tokens = sum(lens)
    other = 4 * (sum(blocks) + case["requests"] * (1 + case["q_heads"]))
    if case["op"] == "sparse":
        scored = sum(max(0, n - FIRST - LAST) for n in blocks if n > case["keep"])
        tokens = sum(n - max(0, b - case["keep"]) * case["block"] for n, b in zip(lens, blocks))
        other += scored * entry + 4 * case["kv_heads"] * sum(min(b, case["keep"]) for b in blocks)
    return {"bytes": 2 * tokens * row + 2 * values * size + other, "flops": 4 * tokens * case["q_heads"] * case["dim"]}


# ---------------------------------------------------------------- the definitions in 64 bits

def _exact_rows(case, page, slot):
    """Rows [n, kv_heads, dim] in 64 bits at `slot` of the raw pages [n, page bytes]."""
    n, heads, dim, block = page.shape[0], case["kv_heads"], case["dim"], case["block"]
    head = torch.arange(heads, device=page.device)

    def byte(at):
        return page.gather(1, at.reshape(n, -1)).to(torch.int64).view(at.shape)
    if case["bits"] == 16:
        at = (slot.view(-1, 1) * heads * dim + torch.arange(heads * dim, device=page.device)) * 2
        word = byte(at) + 256 * byte(at + 1)
        exponent, part = (word >> 7) & 255, word & 127
        value = torch.where(exponent > 0, 1 + part.double() / 128, part.double() / 128) * torch.exp2((exponent.clamp_min(1) - 127).double())
        return torch.where(word >> 15 > 0, -value, value).view(n, heads, dim)

    def small(code, bits, bias):             # 8-bit numbers with that many bits behind the point
        exponent, part = (code >> bits) & (15 if bits == 3 else 3), (code & ((1 << bits) - 1)).double() / (1 << bits)
        value = torch.where(exponent > 0, 1 + part, part) * torch.exp2((exponent.clamp_min(1) - bias).double())
        return torch.where((code >> (7 if bits == 3 else 3)) & 1 > 0, -value, value)
    if case["bits"] == 8:
        at = slot.view(-1, 1) * heads * dim + torch.arange(heads * dim, device=page.device)
        power = byte(block * heads * dim + head * block + slot.view(-1, 1)).double() - 127
        return small(byte(at), 3, 7).view(n, heads, dim) * torch.exp2(power).unsqueeze(-1)
    record = page.shape[1] // heads
    d = torch.arange(dim, device=page.device)
    code = byte(head.view(-1, 1) * record + slot.view(-1, 1, 1) * (dim // 2) + d // 2)
    code = torch.where(d % 2 == 0, code & 15, code >> 4)
    group = byte(head.view(-1, 1) * record + block * dim // 2 + slot.view(-1, 1, 1) * (dim // 16) + d // 16)
    power = byte(head * record + block * (dim // 2 + dim // 16) + slot.view(-1, 1)).double() - 127
    return small(code, 1, 1) * small(group, 3, 7) * torch.exp2(power).unsqueeze(-1)


def _exact_attention(case, q, k, v):
    """(out, lse) of one head's queries [group, dim] over its rows [n, dim], 64 bits."""
    score = (q @ k.T) * case["dim"] ** -0.5
    lse = torch.logsumexp(score, -1)
    return torch.exp(score - lse[:, None]) @ v, lse


def _exact_kept(case, s, r, h, n):
    """Logical blocks that request r's KV head h attends to."""
    if n <= case["keep"]:
        return list(range(n))
    group = case["q_heads"] // case["kv_heads"]
    q = s["q"][r, h * group: (h + 1) * group].double().cpu().numpy()
    u = np.concatenate([np.where(q > 0, q, 0).sum(0), np.where(q < 0, q, 0).sum(0)])
    top, power = np.abs(u).max(), -100
    while top > 32767.0 * 2.0 ** power:
        power += 1
    u = np.rint(u * 2.0 ** -power).astype(np.int64)
    middle = np.arange(FIRST, n - LAST)
    blocks = s["table"][r].cpu().numpy()[middle]
    codes = s["codes"][0, :, h].cpu().numpy().astype(np.int64).reshape(-1, 2 * case["dim"])[blocks]
    scale = s["scales"][0, :, h].cpu().numpy().astype(np.float64)[blocks]
    score = (codes @ u).astype(np.float32).astype(np.float64) * 2.0 ** (scale - 127)
    order = np.lexsort((middle, -score))[: case["keep"] - FIRST - LAST]
    return sorted([*range(FIRST), *middle[order].tolist(), *range(n - LAST, n)])


def exact(case, seed):
    if case["op"] == "bounds":
        return None             # whole numbers, found by comparing and by exact products alone
    s = prepare(case, seed)
    if case["op"] == "append":
        half = case["rotary"] // 2
        pairs = torch.arange(half, device=DEVICE)
        first = pairs if case["layout"] == "half" else 2 * pairs
        second = pairs + half if case["layout"] == "half" else 2 * pairs + 1
        turn = torch.polar(torch.ones(case["tokens"], half, dtype=torch.float64, device=DEVICE),
                           s["positions"].double()[:, None] * s["theta"])[:, None]
        got = []
        for x in (s["q"].double(), s["k"].double()):
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            got.append(x)
        if case["bits"] < 16:
            # a key next to the border of two codes goes either way with the last bit of its rotation, and takes its scales along
            return {"q": got[0], "codes": None, "rows": None, **({"groups": None} if case["bits"] == 4 else {})}
        values = _views(case, s["pages"][0])["values"].double()
        block, slot = s["slots"] // case["block"], s["slots"] % case["block"]
        values[0, block, slot], values[1, block, slot] = got[1], s["v"].double()
        return {"q": got[0], "values": values}
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(case["requests"], case["q_heads"], case["dim"], dtype=torch.float64, device=DEVICE)
    lse = torch.full((case["requests"], case["q_heads"]), -math.inf, dtype=torch.float64, device=DEVICE)
    for r, n in enumerate(_lens(case)):
        if n == 0:
            continue
        at = torch.arange(n, device=DEVICE)
        block, slot = s["table"][r].long()[at // case["block"]], at % case["block"]
        k, v = (_exact_rows(case, s["pages"][0, kv][block], slot) for kv in range(2))
        for h in range(case["kv_heads"]):
            mine = slice(h * group, (h + 1) * group)
            seen = slice(None)
            if case["op"] == "sparse":
                kept = torch.tensor(_exact_kept(case, s, r, h, -(-n // case["block"])), device=DEVICE)
                seen = (at // case["block"]).unsqueeze(-1).eq(kept).any(-1)
            out[r, mine], lse[r, mine] = _exact_attention(case, s["q"][r, mine].double(), k[seen, h], v[seen, h])
    return {"out": out, "lse": lse} if case["op"] == "attend" else {"out": out, "lse": lse, "kept": None, "lens": None}
