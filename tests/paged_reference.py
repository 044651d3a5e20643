"""The paged cache operators from their definitions, in numpy and 64 bits, and the
error bounds that their tests use.  Shares no code with the GPU path."""
import math

import numpy as np

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}   # half a step, relative


def page_tables(cached, new, page, free, head, table, parents=None):
    """(cu, kv_len, slot, position, mask, table, head) for well-formed requests."""
    table = [list(r) for r in table]
    cu, kv_len, slot, position, mask = [0], [], [], [], []
    for b, (c, n) in enumerate(zip(cached, new)):
        for i in range(math.ceil(c / page), math.ceil((c + n) / page)):
            table[b][i] = free[head]
            head += 1
        bits, depth = [], []
        for i in range(n):
            up = (i - 1) if parents is None else parents[b][i]
            bits.append((1 << i) | (bits[up] if up >= 0 else 0))
            depth.append(depth[up] + 1 if up >= 0 else 0)
            slot.append(table[b][(c + i) // page] * page + (c + i) % page)
        position += [c + (d if parents is not None else i) for i, d in enumerate(depth)]
        mask += bits
        cu.append(cu[-1] + n)
        kv_len.append(c + n)
    return cu, kv_len, slot, position, mask, table, head


def rotate(x, position, theta):
    """x [rows, heads, dh], pairs (i, i + dh/2) turned by position * theta^(-2i/dh).
    The angle is reduced to one turn in integers: a fp64 product of a far position keeps
    too few bits behind the point."""
    half = x.shape[-1] // 2
    if theta == 0:
        return x.astype(np.float64)
    rate = [theta ** (-2.0 * i / (2 * half)) / (2 * math.pi) for i in range(half)]
    turns = np.array([[(int(p) * int(r * 2 ** 64) % 2 ** 64) / 2 ** 64 for r in rate] for p in position])
    c, s = np.cos(2 * math.pi * turns)[:, None], np.sin(2 * math.pi * turns)[:, None]
    a, b = x[..., :half].astype(np.float64), x[..., half:].astype(np.float64)
    return np.concatenate([a * c - b * s, b * c + a * s], -1)


def rotate_bound(x, ref, dt):
    """One rounding to dt, and of fp32: the two products, their sum, sine and cosine, and
    an angle off by 2^-23 of half a turn's fraction (at most 2^-23 pi)."""
    half = x.shape[-1] // 2
    mag = np.abs(x[..., :half]) + np.abs(x[..., half:])
    return U[dt] * np.abs(ref) + np.concatenate([mag, mag], -1) * (6 * 2.0 ** -24 + math.pi * 2.0 ** -23)


def attend(q, k, v, seen, dt):
    """One head: q [m, dh], k, v [n, dh], seen [m, n] -> (o, bound on |computed - o|).

    The bound counts: the stored result's rounding (u |o|); the probabilities rounded to
    dt before the product with v (u each, in numerator and sum: 2 u A, A = sum w |v|);
    fp32 scores (a chain of dh products: dh 2^-24 sum |q k|), exponent and exponential
    (2^-22 |s| + 2^-21), each twice again; fp32 sums over the keys (n 2^-24, twice).
    f16 probabilities below its normal range are off by at most 2^-25 each, of a sum that
    is at least 1: in numerator and sum, 2^-25 (sum |v| + n |o|) over the seen keys."""
    q, k, v = (t.astype(np.float64) for t in (q, k, v))
    m, n = q.shape[0], k.shape[0]
    dh = q.shape[1]
    if n == 0:
        return np.zeros((m, dh)), np.zeros((m, dh))
    k0, v0 = np.where(np.isfinite(k), k, 0), np.where(np.isfinite(v), v, 0)
    s = q @ k0.T / math.sqrt(dh)
    s = np.where(seen, s, -np.inf)
    top = s.max(-1, keepdims=True)
    e = np.exp(s - np.where(np.isinf(top), 0, top))
    total = e.sum(-1, keepdims=True)
    w = e / np.where(total == 0, 1, total)
    size = np.where(seen, np.abs(q) @ np.abs(k0).T / math.sqrt(dh), 0).max(-1, keepdims=True)
    u = U[dt]
    rel = 2 * (u if dt != "f32" else 0) + 2 * (dh * 2.0 ** -24 * size + 2.0 ** -22 * size + 2.0 ** -21) + 2 * n * 2.0 ** -24
    o = w @ v0
    small = 2.0 ** -25 * (dt == "f16")
    return o, u * np.abs(o) + rel * (w @ np.abs(v0)) + small * (1 + seen @ np.abs(v0) + seen.sum(-1, keepdims=True) * np.abs(o))


def causal(q, k, v, cu, dt):
    """q [T, hq, dh], k, v [T, hk, dh]; (o, bound) for rows of cu's sequences."""
    g = q.shape[1] // k.shape[1]
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    for a, e in zip(cu[:-1], cu[1:]):
        seen = np.tril(np.ones((e - a, e - a), bool))
        for h in range(q.shape[1]):
            o[a:e, h], bound[a:e, h] = attend(q[a:e, h], k[a:e, h // g], v[a:e, h // g], seen, dt)
    return o, bound


def tree(q, kv, table, page, cu, kv_len, mask, dt):
    """q [T, hq, dh], kv [pool rows, 2, hk, dh]; mask: words per row, or None."""
    g = q.shape[1] // kv.shape[2]
    o, bound = np.zeros(q.shape), np.zeros(q.shape)
    for b, (a, e) in enumerate(zip(cu[:-1], cu[1:])):
        n = e - a
        if n == 0:
            continue
        rows = np.array([table[b][t // page] * page + t % page for t in range(kv_len[b])], int)
        words = mask[a:e] if mask is not None else [(1 << (i + 1)) - 1 for i in range(n)]
        among = np.array([[(int(w) >> j) & 1 for j in range(n)] for w in words], bool)
        seen = np.concatenate([np.ones((n, kv_len[b] - n), bool), among], 1)
        for h in range(q.shape[1]):
            o[a:e, h], bound[a:e, h] = attend(q[a:e, h], kv[rows, 0, h // g], kv[rows, 1, h // g], seen, dt)
    return o, bound
