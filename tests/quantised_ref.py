"""The operators of the 8-bit cache and the verification of drafts restated in numpy and 64 bits, for the GPU tests."""
from __future__ import annotations

import math

import numpy as np


def _value(code: int) -> float:
    sign, e, m = -1.0 if code & 0x80 else 1.0, code >> 3 & 15, code & 7
    if e == 15 and m == 7:
        return math.nan
    return sign * (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))


VALUES = np.array([_value(c) for c in range(256)])           # of every e4m3 code
_SORTED = VALUES[:127]                                         # 0 .. 448, ascending


def encode(x):
    """Codes of values of up to 448 (and more: 448), rounded to nearest, ties to the even code; NaN: 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isnan(x), 0, x)), 448.0)
    hi = np.clip(np.searchsorted(_SORTED, a), 1, 126)
    lo = hi - 1
    d = (a - _SORTED[lo]) - (_SORTED[hi] - a)
    code = np.where((d > 0) | ((d == 0) & (hi % 2 == 0)), hi, lo)
    return np.where(np.isnan(x), 0x7f, code + np.where(np.signbit(x), 128, 0)).astype(np.uint8)


def decode(codes, scale, block):
    """Values of a cache [pages, page, heads, dim] with scales [pages, blocks, heads]."""
    return VALUES[codes] * np.repeat(np.asarray(scale, np.float64), block, 1)[..., None]


_POWERS = 2.0 ** np.arange(-60, 61)


def _least_power(size):
    """Of 2^-60 .. 2^60, the first that is not below each size."""
    return _POWERS[np.minimum(np.searchsorted(_POWERS, size), 120)]


def quantise(codes, scale, rows, slots, block):
    """One layer's keys or values: rows [n, heads, dim] (None: skipped) into slots of codes [pages, page, heads, dim] and scales
    [pages, blocks, heads], both changed in place."""
    pages, page = codes.shape[:2]
    groups = {}
    for x, s in zip(rows, slots):
        if x is not None and 0 <= s < pages * page:
            groups.setdefault(s // block, {})[s % block] = np.asarray(x, np.float64)
    for b, new in groups.items():
        p, first = b * block // page, b * block % page
        stays = [first + i for i in range(max(new)) if i not in new]
        places, x = [first + i for i in new], np.stack(list(new.values()))
        fresh = _least_power(np.where(np.isfinite(x), np.abs(x), 0.0).max((0, 2)) / 448)
        old = scale[p, first // block].astype(np.float64)
        old = np.where((old > 0) & (old < math.inf), old, 0.0)  # (of no use: nothing stays)
        if stays:
            fresh = np.maximum(fresh, _least_power(old))
            for h in np.nonzero(fresh != scale[p, first // block])[0]:
                codes[p, stays, h] = encode(VALUES[codes[p, stays, h]] * (old[h] / fresh[h]))
        codes[p, places] = encode(np.where(np.isfinite(x), x, math.nan) / fresh[None, :, None])
        scale[p, first // block] = fresh


def verify(logits, probs, tokens, parent, cu, temperature, uniform, noise, max_new):
    """path, accepted, next, and of every request how near the nearest decision was (relative)."""
    n, vocab = len(cu) - 1, logits.shape[1]
    path = np.full(logits.shape[0], -1, np.int64)
    accepted, after, margin = np.zeros(n, np.int64), np.full(n, -1, np.int64), np.full(n, np.inf)
    for i in range(n):
        lo, count = int(cu[i]), min(int(cu[i + 1] - cu[i]), max_new)
        if count == 0:
            continue
        greedy = temperature is None or not temperature[i] > 0

        def enter(at):
            x = np.where(np.isnan(logits[lo + at]), -np.inf, logits[lo + at].astype(np.float64))
            top = x.max()
            if top == -np.inf:
                return x, np.zeros(vocab)
            if greedy:
                return x, None
            with np.errstate(invalid="ignore"):
                return x, np.where(x == top, 1.0, np.exp(np.where(x == top, 0.0, x - top) / float(temperature[i])))

        at, path[lo], accepted[i] = 0, lo, 1
        x, w = enter(0)
        e = None if w is None else w.copy()
        q_sum = 0.0
        for j in range(1, count):
            above = j - 1 if parent is None else int(parent[lo + j])
            t = int(tokens[lo + j])
            if above != at or not 0 <= t < vocab:
                continue
            if greedy:
                ok = x.max() > -np.inf and t == int(x.argmax())
            else:
                total = w.sum()
                q = 1.0 if probs is None else float(probs[lo + at, t])
                left, right = float(uniform[lo + j]) * total * q, w[t]
                margin[i] = min(margin[i], abs(left - right) / max(left, right, 1e-300))
                ok = left < right
                if not ok:
                    if probs is None:
                        w[t] = 0.0
                    else:
                        q_sum += total
                        w = np.maximum(e - q_sum * probs[lo + at].astype(np.float64), 0.0)
            if ok:
                at, path[lo + accepted[i]] = j, lo + j
                accepted[i] += 1
                x, w = enter(j)
                e = None if w is None else w.copy()
                q_sum = 0.0
        if greedy:
            after[i] = int(x.argmax()) if x.max() > -np.inf else -1
            continue
        z = noise[i].astype(np.float64)
        for weights in (w, e):
            with np.errstate(divide="ignore", invalid="ignore"):
                r = np.where((weights > 0) & (z > 0), weights / z, 0.0)
            if r.max() > 0:
                after[i] = int(r.argmax())
                two = np.sort(r)[-2:]
                margin[i] = min(margin[i], 1 - two[0] / two[1]) if vocab > 1 else margin[i]
                break
    return path, accepted, after, margin
