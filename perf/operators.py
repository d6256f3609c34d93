"""Cases, plain forms and exact values of the operators that serve a batch of requests from a paged KV cache.

  rope    rotary positions on the query and key heads of a fused QKV buffer (half or interleaved pairs, part of the
          head, scaled frequencies), and the backward direction
  write   K and V rows into pages of bf16 or of e4m3 codes with one power-of-two scale per token and KV head
  read    those pages back into rows
  attend  attention of one new token per request over the pages (ragged contexts, split over their length and joined)

Page layout: [slot][kv_head][dim] values; e4m3 pages end with the scale bytes [kv_head][slot] (2^(byte - 127)),
padded to a multiple of 16.  Where `own` is true, `run` calls the library's operators instead of the plain forms.
"""
import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda" if torch.cuda.is_available() else "cpu"
MIN_EXP, MAX_EXP = -110, 119          # exponents a scale may take
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one token of the 32B shape (64 query and 8 key heads of 128): the resumed decode step
        dict(name="rope-1", op="rope", tokens=1, q_heads=64, kv_heads=8, dim=128, rotary=128, layout="half",
             scaling="none", type="bf16", backward=False, far=4096),
        # a training batch's gradient, half of the head in interleaved pairs, odd length, fp32
        dict(name="rope-back-1003", op="rope", tokens=1003, q_heads=32, kv_heads=8, dim=128, rotary=64,
             layout="interleaved", scaling="linear", type="f32", backward=True, far=32768),
        # a 16k prefix of the 32B shape whose positions go past the trained context
        dict(name="rope-16384", op="rope", tokens=16384, q_heads=64, kv_heads=8, dim=128, rotary=128, layout="half",
             scaling="parts", type="bf16", backward=False, far=1000000),
        # 64 resident requests each append one token (8B / 32B cache: 8 heads of 128)
        dict(name="write-64", op="write", tokens=64, kv_heads=8, dim=128, block=16, elem=1, type="bf16"),
        # a 16k prefix, K and V taken out of the QKV buffer
        dict(name="write-16384", op="write", tokens=16384, kv_heads=8, dim=128, block=16, elem=1, type="bf16"),
        # the gather of a continued prefill: a ragged prefix read back for a chunk's attention
        dict(name="read-577", op="read", tokens=577, kv_heads=2, dim=64, block=16, elem=1, type="f32"),
        # a 16k prefix back into bf16 rows
        dict(name="read-16384", op="read", tokens=16384, kv_heads=8, dim=128, block=16, elem=1, type="bf16"),
        # one short request of the tiny shape: latency
        dict(name="attend-1x161", op="attend", requests=1, ctx=161, q_heads=4, kv_heads=2, dim=64, block=16, elem=2,
             type="f32", lens=1),
        # one long request of the 32B shape over an 8-bit cache: the context has to be split
        dict(name="attend-1x18433", op="attend", requests=1, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16,
             elem=1, type="bf16", lens=2),
        # 16 ragged requests of the 32B shape, bf16 pages
        dict(name="attend-16x8192", op="attend", requests=16, ctx=8192, q_heads=64, kv_heads=8, dim=128, block=16,
             elem=2, type="bf16", lens=3),
        # many short ragged requests of the 8B shape, fp32 queries
        dict(name="attend-128x577", op="attend", requests=128, ctx=577, q_heads=32, kv_heads=8, dim=128, block=16,
             elem=1, type="f32", lens=4),
        # a full server: 32 ragged requests of the 32B shape over an 8-bit cache
        dict(name="attend-32x18433", op="attend", requests=32, ctx=18433, q_heads=64, kv_heads=8, dim=128, block=16,
             elem=1, type="bf16", lens=5),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.5)))))))


def draw(rng):
    op = rng.choice(["rope", "write", "read", "attend", "attend"])
    dim = rng.choice([64, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    kind = rng.choice(["bf16", "f32"])
    if op == "rope":
        return dict(op=op, tokens=_log(rng, 1, 8192), q_heads=kv_heads * rng.choice([1, 2, 4, 8]), kv_heads=kv_heads,
                    dim=dim, rotary=rng.choice([dim, dim // 2, dim - 2 * rng.randint(0, dim // 4)]),
                    layout=rng.choice(["half", "interleaved"]), scaling=rng.choice(["none", "linear", "ntk", "parts"]),
                    type=kind, backward=rng.random() < 0.5, far=_log(rng, 16, 1000000))
    if op in ("write", "read"):
        return dict(op=op, tokens=_log(rng, 1, 16384), kv_heads=kv_heads, dim=dim, block=rng.choice([8, 16, 32]),
                    elem=rng.choice([1, 1, 2]), type=kind)
    requests = _log(rng, 1, 128)
    return dict(op=op, requests=requests, ctx=_log(rng, 1, max(1, min(16384, 250000 // requests))),
                q_heads=kv_heads * rng.choice([1, 2, 4, 8]), kv_heads=kv_heads, dim=dim, block=rng.choice([8, 16, 32]),
                elem=rng.choice([1, 2]), type=kind, lens=rng.randrange(1 << 20))


# ---------------------------------------------------------------- what a program has in hand before the call

def _page_bytes(case):
    values = case["block"] * case["kv_heads"] * case["dim"] * case["elem"]
    return values + (-(-case["block"] * case["kv_heads"] // 16) * 16 if case["elem"] == 1 else 0)


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


def _quantised(x):
    """(codes, scale bytes) of rows: the plain form of what a write does to each row."""
    x = x.float()
    fine = torch.isfinite(x)
    most = torch.where(fine, x.abs(), torch.zeros_like(x)).amax(-1)
    part, power = torch.frexp(most)
    power = (power - 9 + (part > 0.875).int()).clamp(MIN_EXP, MAX_EXP)
    power = torch.where(most > 0, power, torch.full_like(power, MIN_EXP))
    scaled = (x * torch.exp2(-power.float()).unsqueeze(-1)).clamp(-448.0, 448.0)
    scaled = torch.where(fine, scaled, torch.full_like(scaled, math.nan))
    return scaled.to(torch.float8_e4m3fn), (power + 127).to(torch.uint8)


def _views(case, pages):
    """(values [..., block, kv_heads, dim], scale bytes [..., kv_heads, block] or None) of a tensor of pages."""
    lead = pages.shape[:-1]
    n = case["block"] * case["kv_heads"]
    if case["elem"] == 2:
        return pages.view(torch.bfloat16).view(*lead, case["block"], case["kv_heads"], case["dim"]), None
    codes = pages[..., : n * case["dim"]].view(torch.float8_e4m3fn)
    codes = codes.unflatten(-1, (case["block"], case["kv_heads"], case["dim"]))
    return codes, pages[..., n * case["dim"]: n * case["dim"] + n].unflatten(-1, (case["kv_heads"], case["block"]))


def _filled(case, gen, blocks):
    """A pool [1 layer][K, V][blocks][page bytes] of written pages."""
    pages = torch.zeros(1, 2, blocks, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
    values, scales = _views(case, pages)
    rows = _rows(gen, (2, blocks, case["block"], case["kv_heads"], case["dim"]))
    if case["elem"] == 2:
        values[0] = rows.to(torch.bfloat16)
    else:
        codes, powers = _quantised(rows)
        values.view(torch.uint8)[0] = codes.view(torch.uint8)
        scales[0] = powers.transpose(-1, -2)
    return pages


def _theta(case):
    """Frequencies of the rotated pairs, in 64 bits, and the factor on the rotated values."""
    half = case["rotary"] // 2
    base, factor, trained, low, high, gain = 1.0e6, 8.0, 4096.0, 1.0, 32.0, 1.0
    if case["scaling"] == "ntk":
        base *= factor ** (case["rotary"] / (case["rotary"] - 2))
    theta = base ** (-np.arange(half, dtype=np.float64) / half)
    if case["scaling"] == "linear":
        theta = theta / factor
    if case["scaling"] == "parts":
        keep = np.clip((trained * theta / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        theta, gain = (1 - keep) * theta / factor + keep * theta, 0.1 * math.log(factor) + 1.0
    return theta, gain


def prepare(case, seed):
    gen = torch.Generator(device=DEVICE).manual_seed(int(seed))
    state = {"case": case, "own": None}
    if case["op"] == "rope":
        heads = case["q_heads"] + case["kv_heads"]
        width = (case["q_heads"] + 2 * case["kv_heads"]) * case["dim"]
        qkv = torch.randn(case["tokens"], width, generator=gen, device=DEVICE).to(TYPES[case["type"]])
        theta, gain = _theta(case)
        state["x"] = qkv.view(case["tokens"], -1, case["dim"])[:, :heads]       # Q | K of the fused projection
        first = torch.randint(0, max(1, case["far"] - case["tokens"]), (1,), generator=gen, device=DEVICE)
        state["positions"] = (first + torch.arange(case["tokens"], device=DEVICE)).to(torch.int32)
        state["theta"], state["gain"] = torch.from_numpy(theta).to(DEVICE), gain
        state["out"] = torch.empty(case["tokens"], heads, case["dim"], dtype=TYPES[case["type"]], device=DEVICE)
        return state
    if case["op"] in ("write", "read"):
        blocks = -(-case["tokens"] // case["block"]) + 3
        table = torch.randperm(blocks, generator=gen, device=DEVICE)
        at = torch.arange(case["tokens"], device=DEVICE)
        state["slots"] = table[at // case["block"]] * case["block"] + at % case["block"]
        if case["op"] == "read":
            state["pages"] = _filled(case, gen, blocks)
            shape = (case["tokens"], case["kv_heads"], case["dim"])
            state["out"] = [torch.empty(shape, dtype=TYPES[case["type"]], device=DEVICE) for _ in range(2)]
            return state
        state["pages"] = torch.zeros(1, 2, blocks, _page_bytes(case), dtype=torch.uint8, device=DEVICE)
        rows = _rows(gen, (case["tokens"], 4 * case["kv_heads"], case["dim"])).to(TYPES[case["type"]])
        state["k"], state["v"] = rows[:, 2 * case["kv_heads"]: 3 * case["kv_heads"]], rows[:, 3 * case["kv_heads"]:]
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
    return state


# ---------------------------------------------------------------- one pass

def _plain_rope(s):
    case, half, x = s["case"], s["case"]["rotary"] // 2, s["x"]
    angle = s["positions"].double().unsqueeze(-1) * s["theta"]
    cos = (torch.cos(angle) * s["gain"]).float().unsqueeze(1)
    sin = (torch.sin(angle) * (-s["gain"] if case["backward"] else s["gain"])).float().unsqueeze(1)
    part = x[..., : case["rotary"]].float()
    if case["layout"] == "half":
        a, b = part[..., :half], part[..., half:]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    else:
        a, b = part[..., 0::2], part[..., 1::2]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    return torch.cat([turned.to(x.dtype), x[..., case["rotary"]:]], -1)


def _plain_write(s):
    case = s["case"]
    values, scales = _views(case, s["pages"])
    at, slot = s["slots"] // case["block"], s["slots"] % case["block"]
    both = torch.stack([s["k"], s["v"]])
    if case["elem"] == 2:
        values[0, :, at, slot] = both.to(torch.bfloat16)
        return {"values": values}
    codes, powers = _quantised(both)
    values.view(torch.uint8)[0, :, at, slot] = codes.view(torch.uint8)
    scales[0][:, at, :, slot] = powers.transpose(0, 1)
    return {"values": values, "scales": scales}


def _plain_rows(case, pages):
    """Pages [..., page bytes] as fp32 rows [..., block, kv_heads, dim]."""
    values, scales = _views(case, pages)
    if scales is None:
        return values.float()
    return values.float() * torch.exp2(scales.float() - 127.0).transpose(-1, -2).unsqueeze(-1)


def _plain_read(s):
    case = s["case"]
    rows = _plain_rows(case, s["pages"][0][:, s["slots"] // case["block"]])
    slot = (s["slots"] % case["block"]).view(1, -1, 1, 1, 1).expand(2, -1, 1, case["kv_heads"], case["dim"])
    rows = rows.gather(2, slot).squeeze(2).to(TYPES[case["type"]])
    return [rows[0], rows[1]]


def _plain_attend(s):
    case, n = s["case"], s["table"].shape[1] * s["case"]["block"]
    at = s["table"].clamp_min(0).long()
    k = _plain_rows(case, s["pages"][0, 0][at]).flatten(1, 2).permute(0, 2, 1, 3)      # [R, Hkv, n, d]
    v = _plain_rows(case, s["pages"][0, 1][at]).flatten(1, 2).permute(0, 2, 1, 3)
    q = s["q"].float().unflatten(1, (case["kv_heads"], -1)) / math.sqrt(case["dim"])
    score = q @ k.transpose(-1, -2)
    seen = torch.arange(n, device=DEVICE) < s["lens"].unsqueeze(-1)
    score = score.masked_fill(~seen[:, None, None], -math.inf)
    most = score.amax(-1, keepdim=True)
    weight = torch.exp(score - most)
    total = weight.sum(-1, keepdim=True)
    none = (s["lens"] == 0).view(-1, 1, 1)
    out = ((weight @ v) / total).flatten(1, 2).masked_fill(none, 0.0)
    lse = (most + torch.log(total)).flatten(1).masked_fill(none[..., 0], -math.inf)
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _cache(s):
    """The library's cache over the state's pages."""
    import paper_2608_16477_b200 as kv
    from synth.configs import ModelShape
    case = s["case"]
    shape = ModelShape("cache", 1, case["dim"], case["kv_heads"], case["kv_heads"], case["dim"], 8, 1,
                       block_size=case["block"])
    return kv.PagedCache(shape, s["pages"].shape[2], elem_bytes=case["elem"], data=s["pages"])


def _handle(s):
    """What a program keeps beside its inputs: the rotary plan, the cache's descriptor, the attention's scratch."""
    import paper_2608_16477_b200 as kv
    case = s["case"]
    if case["op"] == "rope":
        return kv.Rope(case["rotary"], layout=case["layout"], base=1.0e6, scaling=case["scaling"], factor=8.0,
                       original_ctx=4096, low=1.0, high=32.0, gain=s["gain"])
    cache = _cache(s)
    if case["op"] != "attend":
        return cache, None
    need = kv.kv_paged_attention_batched_scratch_bytes(case["requests"], case["q_heads"], cache, case["ctx"])
    return cache, torch.empty(need, dtype=torch.uint8, device=DEVICE)


def _own(s):
    import paper_2608_16477_b200 as kv
    case = s["case"]
    if s["own"] is None:
        s["own"] = _handle(s)
    if case["op"] == "rope":
        kv.kv_op_rope(s["own"], s["x"], s["positions"], s["out"], backward=case["backward"])
        return s["out"]
    cache, scratch = s["own"]
    if case["op"] == "write":
        kv.kv_op_cache_write(cache, 0, s["k"], s["v"], s["slots"])
        values, scales = _views(case, s["pages"])
        return {"values": values} if scales is None else {"values": values, "scales": scales}
    if case["op"] == "read":
        kv.kv_op_cache_read(cache, 0, s["slots"], s["out"][0], s["out"][1])
        return s["out"]
    kv.kv_op_paged_attention_batched(s["q"], cache, 0, s["table"], s["lens"], case["ctx"], s["out"], scratch,
                                     lse=s["lse"])
    return {"out": s["out"], "lse": s["lse"]}


def run(state):
    if own:
        return _own(state)
    return {"rope": _plain_rope, "write": _plain_write, "read": _plain_read,
            "attend": _plain_attend}[state["case"]["op"]](state)


# ---------------------------------------------------------------- what a pass cannot do without

def work(case):
    size = 2 if case.get("type") == "bf16" else 4
    if case["op"] == "rope":
        values = case["tokens"] * (case["q_heads"] + case["kv_heads"]) * case["dim"]
        turned = values * case["rotary"] // case["dim"]
        return {"bytes": 2 * values * size + 4 * case["tokens"], "flops": 3 * turned}
    row = case["kv_heads"] * (case["dim"] * 2 if case["elem"] == 2 else case["dim"] + 1)      # a token's K or V in a page
    if case["op"] in ("write", "read"):
        rows = 2 * case["tokens"] * case["kv_heads"] * case["dim"]
        return {"bytes": rows * size + 2 * case["tokens"] * row + 8 * case["tokens"], "flops": 3 * rows}
    tokens, values = sum(_lens(case)), case["requests"] * case["q_heads"] * case["dim"]
    tables = sum(-(-n // case["block"]) for n in _lens(case))
    return {"bytes": 2 * tokens * row + 2 * values * size + 4 * (tables + case["requests"] * (1 + case["q_heads"])),
            "flops": 4 * tokens * case["q_heads"] * case["dim"]}


# ---------------------------------------------------------------- the definitions in 64 bits

def _decoded(case, page, slot):
    """Rows [n, kv_heads, dim] in 64 bits at `slot` of the raw pages [n, page bytes]."""
    n, width = page.shape[0], case["kv_heads"] * case["dim"] * case["elem"]
    at = slot.view(-1, 1) * width + torch.arange(width, device=page.device)
    raw = page.gather(1, at).to(torch.int64)
    if case["elem"] == 2:
        bits = raw[:, 0::2] + 256 * raw[:, 1::2]
        exponent, mantissa, negative = (bits >> 7) & 255, bits & 127, bits >> 15
        size, bias = 128, 127
    else:
        exponent, mantissa, negative = (raw >> 3) & 15, raw & 7, raw >> 7
        size, bias = 8, 7
    value = torch.where(exponent > 0, 1 + mantissa.double() / size, mantissa.double() / size)
    value = value * torch.exp2((exponent.clamp_min(1) - bias).double())
    value = torch.where(negative > 0, -value, value).view(n, case["kv_heads"], case["dim"])
    if case["elem"] == 1:
        first = case["block"] * case["kv_heads"] * case["dim"]
        head = torch.arange(case["kv_heads"], device=page.device) * case["block"]
        power = page.gather(1, first + head + slot.view(-1, 1)).double() - 127
        value = value * torch.exp2(power).unsqueeze(-1)
    return value


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "rope":
        theta, gain = _theta(case)
        x, half = s["x"].double(), case["rotary"] // 2
        pairs = torch.arange(half, device=x.device)
        first = pairs if case["layout"] == "half" else 2 * pairs
        second = pairs + half if case["layout"] == "half" else 2 * pairs + 1
        turn = torch.polar(torch.full((case["tokens"], half), gain, dtype=torch.float64, device=x.device),
                           s["positions"].double()[:, None] * torch.from_numpy(theta).to(x.device))
        turned = torch.complex(x[..., first], x[..., second]) * (turn.conj() if case["backward"] else turn)[:, None]
        x[..., first], x[..., second] = turned.real, turned.imag
        return x
    if case["op"] == "write":
        values, scales = _views(case, s["pages"])
        want = values.double()
        powers = None if scales is None else scales.double()
        block, slot = s["slots"] // case["block"], s["slots"] % case["block"]
        for kv, rows in enumerate((s["k"].double(), s["v"].double())):
            if case["elem"] == 2:
                want[0, kv, block, slot] = rows
                continue
            most = rows.abs().amax(-1)
            power = torch.ceil(torch.log2(most / 448.0))
            power = torch.where(most > 448.0 * torch.exp2(power), power + 1, power)
            power = torch.where(most <= 448.0 * torch.exp2(power - 1), power - 1, power).clamp(MIN_EXP, MAX_EXP)
            scaled = rows * torch.exp2(-power).unsqueeze(-1)
            step = torch.exp2(torch.floor(torch.log2(scaled.abs().clamp_min(2.0 ** -6))) - 3)
            want[0, kv, block, slot] = (torch.round(scaled / step) * step).clamp(-448.0, 448.0)
            powers[0, kv][block, :, slot] = power + 127
        return {"values": want} if powers is None else {"values": want, "scales": None}
    if case["op"] == "read":
        block, slot = s["slots"] // case["block"], s["slots"] % case["block"]
        return [_decoded(case, s["pages"][0, kv][block], slot) for kv in range(2)]
    group = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(case["requests"], case["q_heads"], case["dim"], dtype=torch.float64, device=DEVICE)
    lse = torch.full((case["requests"], case["q_heads"]), -math.inf, dtype=torch.float64, device=DEVICE)
    for r, n in enumerate(_lens(case)):
        if n == 0:
            continue
        at = torch.arange(n, device=DEVICE)
        block, slot = s["table"][r].long()[at // case["block"]], at % case["block"]
        k = _decoded(case, s["pages"][0, 0][block], slot).repeat_interleave(group, 1).transpose(0, 1)
        score = torch.einsum("hd,hnd->hn", s["q"][r].double(), k) * case["dim"] ** -0.5
        del k
        v = _decoded(case, s["pages"][0, 1][block], slot).repeat_interleave(group, 1).transpose(0, 1)
        lse[r] = torch.logsumexp(score, -1)
        out[r] = torch.einsum("hn,hnd->hd", torch.exp(score - lse[r][:, None]), v)
    return {"out": out, "lse": lse}
