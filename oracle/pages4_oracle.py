"""fp64 restatement of e2m1 pages, block bounds and the selection of blocks (plain numpy, no code shared with the CUDA path)."""
import math

import numpy as np

from oracle.serving_oracle import e4m3_values

MIN_EXP, MAX_EXP = -110, 116      # range of a row's scale exponent
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
NAN_SCALE = 0x7F


def e2m1_values() -> np.ndarray:
    """Value of every 4-bit code: 1 sign, 2 exponent (bias 1), 1 mantissa bit."""
    return np.concatenate([E2M1, -E2M1])


def quantise_row(x):
    """(codes [d], scale codes [d / 16], scale byte) of one row by the definition, every number found by search."""
    x = np.asarray(x, dtype=np.float64)
    fine = np.isfinite(x)
    most = np.abs(x[fine]).max() if fine.any() else 0.0
    e = MIN_EXP
    while e < MAX_EXP and most > 2688.0 * 2.0 ** e:
        e += 1
    scales = e4m3_values()[:127]
    codes, groups = np.zeros(len(x), np.uint8), np.zeros(len(x) // 16, np.uint8)
    for g in range(len(x) // 16):
        at = slice(16 * g, 16 * g + 16)
        y, ok = np.abs(x[at]) * 2.0 ** -e, fine[at]
        s = 1
        while s < 126 and 6.0 * scales[s] < (y[ok].max() if ok.any() else 0.0):
            s += 1
        groups[g] = s
        if not ok.all():
            groups[g] = NAN_SCALE
            continue
        for i, v in enumerate(y):
            away = np.abs(v - E2M1 * scales[s])
            near = int(np.flatnonzero(away == away.min()).max())      # halves go up
            codes[16 * g + i] = near + (8 if np.signbit(x[16 * g + i]) else 0)
    return codes, groups, e + 127


def decode_row(codes, groups, byte):
    return e2m1_values()[codes] * np.repeat(e4m3_values()[groups], 16) * 2.0 ** (byte - 127.0)


def stored(x):
    """What a row of an e2m1 page holds after x was written."""
    return decode_row(*quantise_row(x))


def page(rows_k, block, record):
    """Bytes [heads * record] of a page from rows [block, heads, d] (None: a slot never written, bytes left 0)."""
    heads, d = next(r for r in rows_k if r is not None).shape
    out = np.zeros((heads, record), np.uint8)
    for s, row in enumerate(rows_k):
        if row is None:
            continue
        for h in range(heads):
            codes, groups, byte = quantise_row(row[h])
            out[h, s * d // 2:(s + 1) * d // 2] = codes[0::2] | codes[1::2] << 4
            out[h, block * d // 2 + s * d // 16:block * d // 2 + (s + 1) * d // 16] = groups
            out[h, block * (d // 2 + d // 16) + s] = byte
    return out.reshape(-1)


# ------------------------------------------------------------------ bounds and selection
INFINITE = 255                    # scale byte of a block that holds what no bound covers


def block_bounds(keys):
    """(codes int8 [2, d], scale byte) of keys [n, d]: dims' maxima rounded up, minima down, in units of the least power of two
    that leaves them within 127."""
    keys = np.asarray(keys, dtype=np.float64)
    most, least = keys.max(0), keys.min(0)
    if not np.isfinite(keys).all() or np.abs(keys).max() > 127 * 2.0 ** 60:
        return np.zeros((2, keys.shape[1]), np.int8), INFINITE
    e = -60
    while np.abs(keys).max() > 127 * 2.0 ** e:
        e += 1
    return np.stack([np.ceil(most * 2.0 ** -e), np.floor(least * 2.0 ** -e)]).astype(np.int8), e + 127


def query_code(q):
    """Whole numbers [2 d] of a group's queries [heads, d]: sums of the positive and of the negative parts, in 15 bits and a sign."""
    q = np.where(np.isfinite(q), np.asarray(q, dtype=np.float64), 0.0)
    u = np.concatenate([np.maximum(q, 0).sum(0), np.minimum(q, 0).sum(0)])
    e = -100
    while np.abs(u).max() > 32767 * 2.0 ** e:
        e += 1
    return np.rint(u * 2.0 ** -e).astype(np.int64)


def select(q, codes, scales, table, n_ctx, block, keep, first, last):
    """(logical blocks kept, ascending; tokens in them) for one request and KV head.  codes [num_blocks, 2, d], scales [num_blocks]."""
    n = -(-n_ctx // block)
    if n <= keep:
        return list(range(n)), n_ctx
    u = query_code(q)
    ranked = []
    for b in range(first, n - last):
        p = table[b]
        if not 0 <= p < len(scales) or scales[p] == INFINITE:
            score = math.inf
        else:
            score = float(np.float32(int(codes[p].astype(np.int64).reshape(-1) @ u))) * 2.0 ** (int(scales[p]) - 127)
        ranked.append((-score, b))
    kept = sorted([b for _, b in sorted(ranked)[:keep - first - last]] + list(range(first)) + list(range(n - last, n)))
    return kept, n_ctx - (n - keep) * block
