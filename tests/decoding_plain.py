"""Plain forms of the 8-bit matrices, the rotation and the draw of a token in 64 bits, written from their definitions (include/enec_lowbit.h,
include/enec_sampling.h), for the tests.  numpy and loops; nothing here is shared with the library."""
import math

import numpy as np
import torch

from lowbit_plain import E4M3, e4m3_encode, product_bound


def exponent_of(a):
    """The least e >= -127 with a <= 448 2^e."""
    e = -127
    if a > 0:
        e = max(-127, math.frexp(a / 448)[1] - 1)
        while a > 448 * 2.0 ** e:
            e += 1
    return e


def fp8_encode(x):
    """codes (rows, padded), scales (rows, padded / 128 up to a multiple of 4) of a float64 matrix."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    full = np.zeros((rows, padded))
    full[:, :cols] = x
    codes, scales = np.zeros((rows, padded), dtype=np.uint8), np.zeros((rows, -(-padded // 512) * 4), dtype=np.uint8)
    for r in range(rows):
        for b in range(padded // 128):
            v = full[r, 128 * b:128 * b + 128]
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            e = exponent_of(np.abs(v).max())
            scales[r, b] = e + 127
            codes[r, 128 * b:128 * b + 128] = e4m3_encode(v * 2.0 ** -e)
    return codes, scales


def fp8_decode(codes, scales, cols):
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))[:, :codes.shape[1] // 128]
    return (E4M3[codes] * np.repeat(power, 128, axis=1))[:, :cols]


def turned(x, first, turns, interleaved):
    """x (tokens, heads, dim), 32-bit values, at positions first, first + 1, ...; each product and sum rounded to 32 bits."""
    half = turns.shape[1]
    out = x.astype(np.float32).copy()
    for t in range(x.shape[0]):
        if first + t < 0:
            out[t] = 0
            continue
        c, s = turns[first + t, :, 0], turns[first + t, :, 1]
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        p, q = x[t][:, a].astype(np.float32), x[t][:, b].astype(np.float32)
        out[t][:, a], out[t][:, b] = p * c - q * s, q * c + p * s
    return out


def draw(l, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, uniform=0.0):
    """(token, logarithm of its probability, its weight) for float64 logits."""
    bad = np.isnan(l).any() or (l == -np.inf).all() or not (0 <= temperature < np.inf) or not (0 <= uniform < 1) or math.isnan(top_p) or math.isnan(min_p)
    if bad:
        return -1, math.nan, 1.0
    order = np.argsort(-l, kind="stable")
    if temperature == 0:
        return int(order[0]), 0.0, 1.0
    largest = l[order[0]]
    w = (l == np.inf).astype(np.float64) if largest == np.inf else np.exp((l - largest) / temperature)
    kept = order[:top_k] if 0 < top_k < l.size else order
    if top_p < 1:
        sums = np.cumsum(w[kept])
        kept = kept[:max(1, int(np.sum(np.concatenate(([0.0], sums[:-1])) < top_p * sums[-1])))]
    kept = np.array([i for n, i in enumerate(kept) if n == 0 or w[i] >= min_p])
    mine = np.zeros(l.size)
    mine[kept] = w[kept]
    sums = np.cumsum(mine)
    token = int(np.sum(sums <= uniform * sums[-1]))
    others = math.fsum(mine[kept]) - mine[token]
    return token, -math.log1p(max(0.0, others) / mine[token]), mine[token]


def products_bound(x, w, y, dtype):
    """How far a product of 8-bit matrices may be from y = x w^T.  lowbit_plain.product_bound, and for 16-bit formats what the 8-bit matrix instructions drop:
    of eight consecutive columns' products each loses less than 2^-13 of a power of two that is at most the largest of them, which itself loses
    nothing: seven times 2^-13 of the largest, for each eight columns."""
    bound = product_bound(x, w, y, dtype)
    if dtype != torch.float32:
        for c in range(0, x.shape[1], 8):
            p = np.abs(x[:, c:c + 8])[:, None] * np.abs(w[:, c:c + 8])[None]
            bound += 7 * 2.0 ** -13 * p.max(-1)
    return bound
