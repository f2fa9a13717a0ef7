"""Plain 64-bit forms, in numpy, of tokens into a cache, means and scores of pages, and their selection."""
import numpy as np

import _fp4_util as F

PAGE, D, DV, ROPE = 64, 576, 512, 64
PAIRS = ROPE // 2


def bf16(x):
    """float -> bf16 bit patterns, to nearest with ties to even (finite numbers)."""
    u = np.ascontiguousarray(x, np.float32).view(np.uint32)
    return ((u + 0x7FFF + ((u >> 16) & 1)) >> 16).astype(np.uint16)


def values(bits):
    return F.bf16_values(bits)


def pairs(interleaved):
    """Columns (of 64) of the first and second members of the 32 pairs."""
    i = np.arange(PAIRS)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + PAIRS)


def places(starts, lens, table, num_blocks):
    """[(token, sequence, position, page or None)] of the tokens that have a sequence and a position in it."""
    out = []
    for b in range(len(lens)):
        for token in range(starts[b], starts[b + 1]):
            at = int(lens[b]) - (int(starts[b + 1]) - token)
            if at < 0:
                continue
            page = int(table[b, at // PAGE]) if at < table.shape[1] * PAGE else -1
            out.append((token, b, at, page if 0 <= page < num_blocks else None))
    return out


def rotate(x, angles, interleaved):
    """x [..., 64], angles [64] -> (rotated, |x cos| + |y sin| of every column)"""
    first, second = pairs(interleaved)
    a, b, c, s = x[..., first], x[..., second], angles[:PAIRS], angles[PAIRS:]
    y, size = np.empty_like(x), np.empty_like(x)
    y[..., first], y[..., second] = a * c - b * s, b * c + a * s
    size[..., first], size[..., second] = abs(a * c) + abs(b * s), abs(b * c) + abs(a * s)
    return y, size


def key(x, angles, weight, eps, interleaved):
    """(the key of a token's 576 numbers, a bound of FP32's error in it).

    The factor: half a step of the mean (2^-24, halved by the root), two of rsqrtf (at most 2 ulp: 2^-22); two products, 2^-24 each: below 2^-21 in all.
    The rotation: a rounding of each product and of their sum, 2^-24 of |x cos| + |y sin| each: 2^-23."""
    y, err = np.empty(D), np.zeros(D)
    y[:DV] = x[:DV]
    if weight is not None:
        y[:DV] = x[:DV] / np.sqrt(np.mean(x[:DV] ** 2) + eps) * weight
        err[:DV] = abs(y[:DV]) * 2.0 ** -21
    y[DV:], size = rotate(x[DV:], angles, interleaved)
    err[DV:] = size * 2.0 ** -23
    return y, err


BF16 = values(np.arange(0x7F80).astype(np.uint16))        # the numbers from 0 up


def rounded(y, grid):
    """The grid's number nearest to y (ties to even), saturating."""
    i = F.nearest(np.minimum(abs(y), grid[-1]), grid)
    return np.copysign(grid[i], y)


def between(got, y, err, grid):
    """Is got a number that something within err of y rounds to?"""
    return (rounded(y - err, grid) <= got) & (got <= rounded(y + err, grid))


def groups_fit(got_codes, got_scales, y, err, kv_scale):
    """4 bits: is every scale one that the group's largest magnitude, and every number one that its quotient by that scale rounds to, within err?  (Two more
    roundings of FP32: of 6 kv_scale and of the quotient, 2^-23.)"""
    g, e = y.reshape(-1, 16) / kv_scale, err.reshape(-1, 16) / kv_scale
    top, slack = abs(g).max(1), e.max(1) + abs(g).max(1) * 2.0 ** -22
    scale = F.e4m3(got_scales.reshape(-1))
    ok = (rounded((top - slack) / 6, F.E4M3) <= scale) & (scale <= rounded((top + slack) / 6, F.E4M3))
    nibble = np.stack([got_codes & 15, got_codes >> 4], -1).reshape(-1, 16)
    v = F.E2M1[nibble & 7] * np.where(nibble & 8, -1.0, 1.0)
    step = np.where(scale > 0, scale, 1.0)[:, None]
    q, qe = g / step, e / step + abs(g / step) * 2.0 ** -23
    return ok & np.where(scale[:, None] > 0, between(v, q, qe, F.E2M1), v == 0).all(1)


def seen(n, Sq, t, width):
    return max(0, min(int(n), width * PAGE) - Sq + t + 1)


def pages_of(n):
    return (n + PAGE - 1) // PAGE


def scores(q, means, table, lens, scale):
    """q float64 [B, Sq, H, 576], means float64 [blocks, 576] -> (scores [B, Sq, W], a bound of their relative error)."""
    B, Sq, H, _ = q.shape
    W = table.shape[1]
    out, bound = np.zeros((B, Sq, W)), np.zeros((B, Sq))
    for b in range(B):
        m = np.where(((table[b] >= 0) & (table[b] < len(means)))[:, None], means[np.clip(table[b], 0, len(means) - 1)], 0.0)
        for t in range(Sq):
            n = seen(lens[b], Sq, t, W)
            count = (n - 1) // PAGE if n > 0 else 0
            if count == 0:
                continue
            logits = q[b, t] @ m[:count].T * scale
            p = np.exp(logits - logits.max(1, keepdims=True))
            out[b, t, :count] = (p / p.sum(1, keepdims=True)).sum(0)
            # 576 products, exact, added up in FP32 by an adder that may truncate: 2^-23 of their magnitudes' sum each; what 2^x of FP32 arguments loses
            # (a logit's own rounding among it), the sums over pages and heads: 2^-20 and 2^-23 for each of their roundings, in pieces of at most 64 and 128
            size = (abs(q[b, t]) @ abs(m[:count]).T * abs(scale)).max()
            bound[b, t] = 2 * size * 576 * 2.0 ** -23 + (2 * abs(logits).max() + 256 + count / 64) * 2.0 ** -22
    return out, bound


def select(scores, lens, keep, sink, recent, Sq, width):
    """[positions of the pages] and the number of keys, for every row (b, t)."""
    B = len(lens)
    out = []
    for b in range(B):
        for t in range(Sq):
            n = seen(lens[b], Sq, t, width)
            count = pages_of(n)
            if count <= keep:
                out.append((list(range(count)), n))
                continue
            ends = list(range(sink)) + list(range(count - recent, count))
            s = np.where(np.isnan(scores[b, t]), -np.inf, scores[b, t])
            others = sorted(range(sink, count - recent), key=lambda p: (-s[p], p))[: keep - sink - recent]
            out.append((sorted(ends + others), n - (count - keep) * PAGE))
    return out
