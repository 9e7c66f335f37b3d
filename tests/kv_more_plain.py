"""Rotation by position, the 4-bit cache and blocks' summaries of include/pag.h in numpy and 64 bits, as plainly as they can be said."""
import numpy as np

import kv_plain as plain

FP4 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def encode_fp4(y):
    """Codes of numbers that are already divided by their power of two: the nearest, of two equally near ones the even code."""
    a = np.abs(np.where(np.isnan(y), 0.0, np.clip(y, -6.0, 6.0)))
    far = np.abs(a[..., None] - FP4)
    nearest = far == far.min(-1, keepdims=True)
    even = nearest & (np.arange(8) % 2 == 0)
    code = np.where(even.any(-1), even.argmax(-1), nearest.argmax(-1))
    return (code | np.where(np.signbit(y) & (code > 0), 8, 0)).astype(np.uint8)


def decode_fp4(code):
    return np.where(code & 8, -1.0, 1.0) * FP4[code & 7]


def least_exponent_fp4(most):
    e = -64
    while most > 7.0 * 2.0 ** e:
        e += 1
    return e


def shapes(pages, heads, page, dim, fmt):
    width = -(-dim // 64) * 64
    if fmt == "fp4":
        return (pages, heads, page, 2, width // 2), (pages, heads, page // 16, 2, width // 32, 16)
    return (pages, heads, page, 2, width), (pages, heads, page // 16, 2)


def append(data, exponents, dim, fmt, k, v, slots):
    """In place, any format; k and v [tokens, heads, dim] float64."""
    if fmt != "fp4":
        return plain.append(data, exponents, dim, fmt, k, v, slots)
    pages, heads, page = data.shape[:3]
    width = data.shape[4] * 2
    for i, slot in enumerate(slots):
        if not 0 <= slot < pages * page:
            continue
        p, t = slot // page, slot % page
        for kind, x in ((0, k), (1, v)):
            for h in range(heads):
                row = np.zeros(width)
                row[:dim] = x[i, h]
                codes = np.zeros(width, np.uint8)
                for b in range(width // 32):
                    part = row[32 * b:32 * b + 32]
                    finite = np.abs(part[np.isfinite(part)])
                    e = least_exponent_fp4(finite.max() if finite.size else 0.0)
                    codes[32 * b:32 * b + 32] = encode_fp4(part * 2.0 ** -e)
                    exponents[p, h, t // 16, kind, b, t % 16] = e
                data[p, h, t, kind] = codes[0::2] | codes[1::2] << 4


def numbers(data, exponents, dim, fmt):
    """-> [pages, heads, page, 2, dim]"""
    if fmt != "fp4":
        return plain.numbers(data, exponents, dim, fmt)
    codes = np.stack([data & 15, data >> 4], -1).reshape(*data.shape[:-1], -1)[..., :dim]
    e = exponents.astype(np.float64).transpose(0, 1, 2, 5, 3, 4)                     # [pages, heads, blocks, 16, 2, parts]
    e = np.repeat(e.reshape(*data.shape[:4], -1), 32, -1)[..., :dim]
    return decode_fp4(codes) * 2.0 ** e


def turn(x, positions, frequencies, pairs):
    """Rows [tokens, heads, dim] float64; frequencies float32."""
    n = 2 * len(frequencies)
    angle = np.asarray(positions, np.float64)[:, None, None] * frequencies.astype(np.float64)
    c, s = np.cos(angle), np.sin(angle)
    out = x.copy()
    first, second = (slice(0, n // 2), slice(n // 2, n)) if pairs == "halves" else (slice(0, n, 2), slice(1, n, 2))
    out[..., first] = x[..., first] * c - x[..., second] * s
    out[..., second] = x[..., second] * c + x[..., first] * s
    return out


def rounded(x, dtype):
    """The nearest numbers of a type, as float64: 8, 11 or 24 bits, of two equally near ones the even one."""
    bits, least = {"bf16": (8, -126), "fp16": (11, -14), "fp32": (24, -126)}[dtype]
    _, e = np.frexp(x)
    step = 2.0 ** (np.maximum(e - 1, least) - (bits - 1)).astype(np.float64)
    return np.rint(x / step) * step


def summary(keys):
    """keys [tokens, dim] -> (largest, smallest) as integers [2, dim], and their exponent."""
    hi, lo = keys.max(0), keys.min(0)
    e = plain.least_exponent(max(np.abs(hi).max(), np.abs(lo).max()), "int8")
    return np.stack([np.ceil(hi * 2.0 ** -e), np.floor(lo * 2.0 ** -e)]), e


def query_codes(q):
    """A row of q -> integers and their exponent."""
    finite = np.abs(q[np.isfinite(q)])
    e = plain.least_exponent(finite.max() if finite.size else 0.0, "int8")
    return plain.encode(q * 2.0 ** -e, "int8").view(np.int8).astype(np.float64), e


def select(scores, k):
    """scores: (block, score) of those that may be chosen -> the k best, ascending, -1 behind them."""
    best = sorted(sorted(scores, key=lambda x: (-x[1], x[0]))[:k])
    return [b for b, _ in best] + [-1] * (k - len(best))
