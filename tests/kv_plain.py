"""The cache, the block tables and the attention of include/pag.h in numpy and 64 bits, as plainly as they can be said."""
import math

import numpy as np

LARGEST = {"int8": 127.0, "fp8": 448.0}


def fp8_numbers():
    """What the 256 codes with 4 exponent and 3 mantissa bits stand for."""
    out = np.empty(256)
    for code in range(256):
        sign, e, f = (-1.0 if code & 128 else 1.0), (code >> 3) & 15, code & 7
        out[code] = sign * (f / 8 * 2.0 ** -6 if e == 0 else (1 + f / 8) * 2.0 ** (e - 7))
        if code & 127 == 127:
            out[code] = math.nan
    return out


_FP8 = fp8_numbers()


def decode(codes, fmt):
    return codes.view(np.int8).astype(np.float64) if fmt == "int8" else _FP8[codes]


def encode(y, fmt):
    """Codes of numbers that are already divided by their power of two."""
    y = np.where(np.isnan(y), 0.0, np.clip(y, -LARGEST[fmt], LARGEST[fmt]))
    if fmt == "int8":
        return np.rint(y).astype(np.int8).view(np.uint8)
    numbers = _FP8[:127]                                  # ascending
    a = np.abs(y)
    hi = np.clip(np.searchsorted(numbers, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    down, up = a - numbers[lo], numbers[hi] - a
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    return (code | np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def least_exponent(most, fmt):
    e = -64
    while most > LARGEST[fmt] * 2.0 ** e:
        e += 1
    return e


def append(data, exponents, dim, fmt, k, v, slots):
    """In place.  data [pages, heads, page, 2, width], exponents [pages, heads, page / 16, 2], k and v [tokens, heads, dim] float64."""
    pages, heads, page = data.shape[:3]
    i = 0
    while i < len(slots):
        if not 0 <= slots[i] < pages * page:
            i += 1
            continue
        block = slots[i] // 16
        j = i
        while j < len(slots) and 0 <= slots[j] < pages * page and slots[j] // 16 == block:
            j += 1
        p, first = block * 16 // page, block * 16 % page
        places = [int(s) % 16 for s in slots[i:j]]
        for h in range(heads):
            for kind, x in ((0, k), (1, v)):
                new = x[i:j, h]
                finite = np.abs(new[np.isfinite(new)])
                e = least_exponent(finite.max() if finite.size else 0.0, fmt)
                held = int(exponents[p, h, first // 16, kind])
                rows = data[p, h, first:first + 16, kind]
                if 0 in places:
                    for r in range(16):
                        if r not in places:
                            rows[r] = 0
                else:
                    e = max(e, held)
                    if e > held:
                        for r in range(16):
                            if r not in places:
                                rows[r] = encode(decode(rows[r], fmt) * 2.0 ** (held - e), fmt)
                for r, row in zip(places, new):
                    rows[r] = 0
                    rows[r, :dim] = encode(row * 2.0 ** -e, fmt)
                exponents[p, h, first // 16, kind] = e
        i = j


def numbers(data, exponents, dim, fmt):
    """-> [pages, heads, page, 2, dim]"""
    e = np.repeat(exponents.astype(np.float64), 16, axis=2)
    return decode(data[..., :dim], fmt) * 2.0 ** e[..., None]


def attend_row(q, keys, values, scale, softcap=0.0, slope=0.0, distance=None):
    """One row over n keys -> out [dim], lse, sum of weight times |value| [dim], largest sum of |products| of a score."""
    if len(keys) == 0:
        return np.zeros(values.shape[1]), -math.inf, np.zeros(values.shape[1]), 0.0
    s = scale * (keys @ q)
    if softcap:
        s = softcap * np.tanh(s / softcap)
    if slope:
        s = s - slope * distance
    m = s.max()
    p = np.exp(s - m)
    total = p.sum()
    p /= total
    return p @ values, m + math.log(total), p @ np.abs(values), float((np.abs(keys) @ np.abs(q)).max() * abs(scale))


def tolerance(dim, dtype_bits, out, spread, products, softcap=0.0, slope_reach=0.0):
    """How far out and lse may be off.

    A score sums `dim` products in 32 bits (dim * 2^-24 of the sum of their magnitudes at worst) and takes a few roundings of its own
    size after that (tanh and exp2 are good to 2^-22 of their scale: the cap, the largest exponent); a weight is off by that and by its
    rounding to a 16-bit float with 11 bits, 2^-11; the sums of weights and of products are off by 2^-20 at the lengths tested.
    out is rounded to its own type: 2^-8 (8 bits) or 2^-11 (11 bits) of itself, with subnormals below 2^-14 in the latter."""
    score = dim * 2.0 ** -24 * products + 2.0 ** -21 * (products + softcap + slope_reach) + 2.0 ** -20
    o = (2.0 ** -11 + 2 * score) * spread + np.abs(out) * 2.0 ** -dtype_bits + 2.0 ** -24
    return o, score * 2


def extend(lengths, table, free_pages, free_count, add, page, total):
    """-> dict of what pag_kv_extend writes; table is changed in place."""
    n, width = table.shape
    offsets, context, granted, after = [0], [], [], []
    slots, positions, requests = [], [], []
    taken, wanted = 0, 0
    for r in range(n):
        length, a = int(lengths[r]), max(int(add[r]), 0)
        have, need = -(-length // page), -(-(length + a) // page) - -(-length // page)
        fits = have + need <= width
        if fits:
            wanted += need
        ok = fits and (need == 0 or wanted <= free_count)
        if ok and need:
            for i in range(need):
                table[r, have + i] = free_pages[free_count - 1 - (wanted - need) - i]
            taken = wanted
        granted.append(int(ok))
        after.append(length + a if ok else length)
        context.append(length + a if ok else 0)
        offsets.append(offsets[-1] + a)
        for i in range(a):
            p = length + i
            slots.append(int(table[r, p // page]) * page + p % page if ok else -1)
            positions.append(p if ok else -1)
            requests.append(r)
    pad = total - len(slots)
    if pad < 0:
        slots, positions, requests = slots[:total], positions[:total], requests[:total]
    else:
        slots, positions, requests = slots + [-1] * pad, positions + [-1] * pad, requests + [-1] * pad
    return dict(offsets=offsets, context=context, granted=granted, lengths=after, free_count=[free_count - taken], slots=slots,
                positions=positions, requests=requests)
