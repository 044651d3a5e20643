"""The operators of a paged cache under a budget from their definitions, in numpy and 64 bits
(angles in integers), and the error bounds that their tests use.  Shares no code with the GPU
path."""
import math

import numpy as np

U = {"bf16": 2.0 ** -8, "f16": 2.0 ** -11, "f32": 2.0 ** -24}   # half a step, relative


def rates(theta, rd, scaling="none", factor=1.0, low=1.0, high=1.0, length=1):
    """Radians per position of each pair."""
    out = []
    first = last = 0.0
    if scaling == "pairs":
        first, last = (rd * math.log(length / (n * 2 * math.pi)) / (2 * math.log(theta)) for n in (high, low))
        first, last = max(math.floor(first), 0), min(math.ceil(last), rd - 1)
        if last <= first:
            last = first + 0.001
    for i in range(rd // 2):
        r = theta ** (-2.0 * i / rd)
        share = 1.0                                   # of the rate that is kept as it is
        if scaling == "linear":
            share = 0.0
        elif scaling == "turns":
            share = (length * r / (2 * math.pi) - low) / (high - low)
        elif scaling == "pairs":
            share = 1 - (i - first) / (last - first)
        share = min(max(share, 0.0), 1.0)
        out.append(r * (share + (1 - share) / factor))
    return out


def turn(x, position, rate, interleaved, magnitude=1.0):
    """x [rows, heads, dh]; the first 2 len(rate) values of a head turn.  An angle is reduced to one
    turn in integers: a fp64 product of a far position keeps too few bits behind the point."""
    half, rd = len(rate), 2 * len(rate)
    part = [int(r / (2 * math.pi) * 2 ** 64) for r in rate]
    turns = np.array([[(int(p) * k % 2 ** 64) / 2 ** 64 for k in part] for p in position]).reshape(len(position), half)
    c, s = magnitude * np.cos(2 * math.pi * turns)[:, None], magnitude * np.sin(2 * math.pi * turns)[:, None]
    out = x.astype(np.float64).copy()
    first, second = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, half), slice(half, rd))
    a, b = out[..., first].copy(), out[..., second].copy()
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    return out


def turn_bound(x, ref, position, rd, interleaved, dt, magnitude=1.0):
    """One rounding to dt of what turns (the rest is copied); of fp32: sine and cosine and their product
    with the magnitude, the two products and their sum; an angle off by 2^-23 of half a turn, and by a
    rate off by 2^-50 of itself (at most one radian) times the position."""
    half = rd // 2
    bound = np.zeros(ref.shape)
    first, second = (slice(0, rd, 2), slice(1, rd, 2)) if interleaved else (slice(0, half), slice(half, rd))
    mag = abs(magnitude) * (np.abs(x[..., first]) + np.abs(x[..., second]))
    angle = math.pi * 2.0 ** -23 + np.abs(np.asarray(position, float))[:, None, None] * 2.0 ** -50
    for part in (first, second):
        bound[..., part] = U[dt] * np.abs(ref[..., part]) + mag * (8 * 2.0 ** -24 + angle)
    return bound


def mass(q, keys, table, page, requests, keep, mass_in, head_dim):
    """q [T, hq, dh], keys [pool rows, hk, dh]; requests: per request (rows of q that look, their new-row
    numbers, n, kv_len).  Returns per request (weights [kv_len], bound).

    The bound counts, relative to each weight: fp32 scores (a chain of dh products: dh 2^-24 sum |q k|),
    exponent and exponential (2^-22 |s| + 2^-21), in numerator and sum; the sum over the keys and its
    reciprocal (n + 4) 2^-24; and of the sum over columns one rounding a term.  What came in is
    multiplied and added once."""
    g = q.shape[1] // keys.shape[1]
    out = []
    for b, (rows, places, n, kv) in enumerate(requests):
        at = np.array([table[b][t // page] * page + t % page for t in range(kv)], int)
        c = kv - n
        w, err = np.zeros(kv), np.zeros(kv)
        for h in range(q.shape[1]):
            for r, i in zip(rows, places):
                seen = c + i + 1
                k = keys[at[:seen], h // g].astype(np.float64)
                s = k @ q[r, h].astype(np.float64) / math.sqrt(head_dim)
                size = np.abs(k) @ np.abs(q[r, h].astype(np.float64)) / math.sqrt(head_dim)
                with np.errstate(invalid="ignore"):
                    e = np.exp(s - s.max())
                    p = e / e.sum()
                w[:seen] += p
                err[:seen] += p * (2 * (head_dim * 2.0 ** -24 * size.max() + 2.0 ** -22 * size.max() + 2.0 ** -21) + (seen + 4) * 2.0 ** -24)
        columns = q.shape[1] * max(len(rows), 1)
        old = keep * np.asarray(mass_in[b][:c], np.float64) if keep != 0 else np.zeros(c)
        err += w * (columns + 1) * 2.0 ** -24
        w[:c] += old
        err[:c] += 2 * np.abs(old) * 2.0 ** -24
        out.append((w, err))
    return out


def select(mass, birth, kv_len, gone, budget, sinks, recent):
    """One request: (K, gone out, moving rows, their places)."""
    k = min(budget, kv_len)
    young = kv_len + gone - min(recent, k)

    def key(t):
        if birth[t] >= young:
            return (0, 0.0, t)
        if birth[t] < sinks:
            return (1, 0.0, t)
        return (2, 0.0, t) if math.isnan(mass[t]) else (3, -float(mass[t]), t)

    kept = set(sorted(range(kv_len), key=key)[:k])
    return k, gone + kv_len - k, [t for t in range(k, kv_len) if t in kept], [t for t in range(k) if t not in kept]
