"""Plain forms of the low-bit operators in 64 bits, written from their definitions (include/enec_lowbit.h), for the tests.
numpy and loops; nothing here is shared with the library."""
import math

import numpy as np
import torch

E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=np.float64)
UNIT = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}      # largest relative error of one rounding
LEAST = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25, torch.float32: 2.0 ** -150}  # half the smallest positive value


def e4m3_values():
    """The values of the 256 E4M3 codes: sign, 4 bits of exponent (bias 7), 3 of mantissa, all ones = NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = c >> 3 & 15, c & 7
        a = math.nan if (e, m) == (15, 7) else m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)
        v[c] = -a if c & 128 else a
    return v


E4M3 = e4m3_values()


def nearest(x, values):
    """Index of the value nearest to |x| in an ascending list, ties to the even index, beyond the last one the last one."""
    x = np.abs(x)
    hi = np.clip(np.searchsorted(values, x), 0, len(values) - 1)
    lo = np.maximum(hi - 1, 0)
    below, above = x - values[lo], values[hi] - x
    return np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)


def e4m3_encode(x):
    """Codes of finite values (NaN: a NaN code)."""
    i = nearest(np.nan_to_num(x), E4M3[:127])
    i = np.where(np.isnan(x), 127, i)
    return (i + 128 * np.signbit(x)).astype(np.uint8)


def mx4_encode(x):
    """codes (rows, padded / 2), scales (rows, padded / 32) of a float64 matrix."""
    rows, cols = x.shape
    padded = -(-cols // 128) * 128
    full = np.zeros((rows, padded))
    full[:, :cols] = x
    codes = np.zeros((rows, padded), dtype=np.uint8)
    scales = np.zeros((rows, padded // 32), dtype=np.uint8)
    for r in range(rows):
        for b in range(padded // 32):
            v = full[r, 32 * b:32 * b + 32]
            a = np.abs(v).max()
            if not np.isfinite(v).all():
                scales[r, b] = 255
                continue
            byte = 0 if a == 0 else max(0, math.frexp(a)[1] - 1 - 2 + 127)
            scales[r, b] = byte
            codes[r, 32 * b:32 * b + 32] = nearest(v * 2.0 ** (127 - byte), E2M1) + 8 * np.signbit(v)
    return codes[:, 0::2] | codes[:, 1::2] << 4, scales


def mx4_decode(codes, scales, cols):
    index = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)
    values = np.concatenate((E2M1, -E2M1))[index]
    power = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    return (values * np.repeat(power, 32, axis=1))[:, :cols]


def rounded(x, dtype):
    """float64 values that have at most 24 bits, rounded once to a torch format."""
    return torch.from_numpy(np.asarray(x, dtype=np.float64).astype(np.float32)).to(dtype)


def product_bound(x, w, y, dtype):
    """How far a product may be from y = x w^T: one rounding to the format, and a relative error of 2^-23 for each addition in 32
    bits (twice what an addition to nearest makes) of the terms' magnitudes."""
    k = x.shape[1]
    return UNIT[dtype] * np.abs(y) + LEAST[dtype] + (k + 8) * 2.0 ** -23 * (np.abs(x) @ np.abs(w).T)


class PlainCache:
    """The cache as a dictionary: (page, head, slot) values by codes and a scale exponent for each (page, head), keys or values."""

    def __init__(self, page, heads, dim):
        self.page, self.heads, self.dim = page, heads, dim
        self.codes, self.exponent = {}, {}

    def write(self, x, table, starts, lengths):
        for b in range(len(lengths)):
            new = starts[b + 1] - starts[b]
            first = lengths[b] - new
            for slot in range(max(0, first) // self.page, -(-lengths[b] // self.page)):
                lo, hi = max(first, slot * self.page), min(lengths[b], (slot + 1) * self.page)
                if lo < 0:
                    lo = 0
                if lo >= hi:
                    continue
                p = int(table[b][slot])
                fresh = x[starts[b] + lo - first:starts[b] + hi - first]
                for h in range(self.heads):
                    v = fresh[:, h]
                    a = np.abs(np.where(np.isfinite(v), v, 0)).max()
                    e = -127
                    if a > 0:
                        e = max(-127, math.ceil(math.log2(a / 448)) - 1)
                        while a > 448 * 2.0 ** e:
                            e += 1
                    if lo > slot * self.page:
                        old = self.exponent[p, h]
                        if old >= e:
                            e = old
                        else:
                            for i in range(lo - slot * self.page):
                                self.codes[p, h, i] = e4m3_encode(E4M3[self.codes[p, h, i]] * 2.0 ** (old - e))
                    self.exponent[p, h] = e
                    for i in range(lo, hi):
                        c = np.clip(v[i - lo] * 2.0 ** -e, -448, 448)
                        self.codes[p, h, i - slot * self.page] = e4m3_encode(np.where(np.isnan(v[i - lo]), np.nan, c))

    def read(self, table, length):
        """(length, heads, dim) values of a sequence."""
        out = np.zeros((length, self.heads, self.dim))
        for t in range(length):
            p = int(table[t // self.page])
            for h in range(self.heads):
                out[t, h] = E4M3[self.codes[p, h, t % self.page]] * 2.0 ** self.exponent[p, h]
        return out


def attention(q, k, v, scale, dtype):
    """Outputs of the newest tokens q (new, q_heads, dim) over keys and values (length, heads, dim), and how far computed ones may be
    off.  A computed score is off by at most (dim + 8) 2^-23 of its terms' magnitudes and 2^-22 of itself (scaling, maximum), an
    exponential by 2^-21 of itself; weights are rounded to bf16 (fp16 tensors: to two bf16 numbers), sums over n tokens add
    n 2^-23, and all these errors come in the numerator and in the sum that it is divided by."""
    new, heads, dim = q.shape
    length, group = k.shape[0], q.shape[1] // k.shape[1]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(new):
        n = length - new + i + 1
        if n <= 0:
            continue
        for h in range(heads):
            kk, vv = k[:n, h // group], v[:n, h // group]
            s = kk @ q[i, h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[i, h] = w @ vv
            terms = np.abs(kk) @ np.abs(q[i, h]) * abs(scale)
            e = ((dim + 8) * 2.0 ** -23 * terms + 2.0 ** -22 * np.abs(s) + 2.0 ** -21).max() + (n + 8) * 2.0 ** -23
            weight = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -16
            bound[i, h] = UNIT[dtype] * np.abs(out[i, h]) + LEAST[dtype] + (weight + 3 * e) * (w @ np.abs(vv))
    return out, bound
