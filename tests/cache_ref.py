"""Plain 64-bit forms of the 8-bit cache and of block-selected attention, for the tests (numpy, CPU).

Error bounds.  A rounding to a type is off by at most half a step, eps / 2 relative (bf16 2^-8, fp16 2^-11, fp32 2^-24).
The attention kernels differ from the exact value by
  * logits: products are exact, 128 fp32 additions, the factor's two roundings, and the fp16 image of the query
    (exact to 2^-25 of its largest element):  e = s (131 * 2^-24 sum|q k| + 2^-25 max|q| sum|k|), s = 128^-1/2;
  * weights: exp2 to 2^-21, one rounding to fp16 (2^-11) for rows of whole blocks of the 8-bit cache, two to bf16 (2^-16
    together) for bf16 rows (weights_bf16 grants one in the numerator and one in the sum that divides it, 2^-8 each;
    `attend_few` what they have), nothing smaller than 2^-31 of the largest weight kept by fp16;
  * a sum of n fp32 terms in partial sums of at most 4096: 2^-12 relative is generous for n <= 2^17;
  * the result's rounding to bf16: 2^-8 |y|, and half a step of its subnormals, 2^-134.
With A = sum_i p_i |v_i| (p normalised) the first two give (2 e + 2^-20 + w) A, w = 2^-11 or 2 * 2^-8.
"""
import math

import numpy as np

TOP = {"e4m3": (448.0, 3, -6), "e5m2": (57344.0, 2, -14)}
S = 128 ** -0.5


def scale_of(amax, top):
    """2^max(ceil(log2(amax / top)), -126), exactly."""
    amax = np.asarray(amax, np.float64)
    e = np.full(amax.shape, -126, np.int64)
    for i in np.ndindex(amax.shape):
        if amax[i] > 0:
            k = int(math.ceil(math.log2(amax[i] / top)))
            while amax[i] > top * 2.0 ** k:
                k += 1
            while amax[i] <= top * 2.0 ** (k - 1):
                k -= 1
            e[i] = max(k, -126)
    return np.exp2(e.astype(np.float64))


def round_code(x, fmt):
    """Nearest representable code value, ties to even."""
    _, bits, lowest = TOP[fmt]
    _, e = np.frexp(x)
    step = np.exp2(np.maximum(e - 1, lowest).astype(np.float64) - bits)
    return np.rint(x / step) * step


def quantise(rows, fmt):
    """[16][128] -> (code values [16][128], scale)."""
    s = float(scale_of(np.abs(rows).max(), TOP[fmt][0]))
    return round_code(rows / s, fmt), s


def block_bounds(rows):
    """[1..16][128] -> (int8 [2][128], scale)."""
    both = np.stack([rows.min(0), rows.max(0)])
    s = float(scale_of(np.abs(both).max(), 127.0))
    return np.rint(both / s).astype(np.int8), s


def query_codes(q):
    s = float(scale_of(np.abs(q).max(), 127.0))
    return np.rint(q / s).astype(np.int64), s


def block_scores(q, codes, scales):
    """q [128], codes int8 [n][2][128], scales [n] -> [n]."""
    q8, qs = query_codes(q)
    c = codes.astype(np.int64)
    return np.maximum(q8 * c[:, 0], q8 * c[:, 1]).sum(-1) * scales * qs


def select_blocks(score, nb, top, sink, recent):
    lo = min(sink, nb)
    hi = max(lo, nb - recent)
    order = sorted(range(lo, hi), key=lambda j: (-score[j], j))[:top]
    return list(range(lo)) + sorted(order) + list(range(hi, nb))


def attend(q, k, v, weights_bf16):
    """(y, lse, bound on |y|'s error [128], bound on the lse's error) over rows k, v [n][128]; n = 0: zeros, -inf."""
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    if len(k) == 0:
        return np.zeros(128), -math.inf, np.zeros(128), 0.0
    a = k @ q * S
    m = a.max()
    p = np.exp(a - m)
    total = p.sum()
    p /= total
    y = p @ v
    e = float((S * (131 * 2.0 ** -24 * (np.abs(k) @ np.abs(q)) + 2.0 ** -25 * np.abs(q).max() * np.abs(k).sum(-1))).max())
    big = p @ np.abs(v)
    w = 2 * 2.0 ** -8 if weights_bf16 else 2.0 ** -11
    tol = 2.0 ** -8 * np.abs(y) + (2 * e + 2.0 ** -20 + 2.0 ** -12 + w) * big + len(k) * 2.0 ** -31 * p.max() * np.abs(v).max() + 2.0 ** -134
    lse = m + math.log(total)
    return y, lse, tol, e + 2.0 ** -20 + 2.0 ** -12 * (len(k) > 4096) + 2.0 ** -22 * abs(lse)


def attend_few(q, k, v, weight):
    """(y, lse, bound, bound on the lse's error) as `attend` gives them, for at most a few hundred rows: the sums counted term by
    term (n roundings of 2^-23, numerator and divisor, a matrix product's included), and weights that enter the product to `weight`
    relative ([n] or one number) while the divisor sums them as they are in fp32."""
    y, lse, _, _ = attend(q, k, v, True)
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    if len(k) == 0:
        return y, lse, np.zeros(128), 0.0
    p = np.exp(k @ q * S - lse)
    e = float((S * (131 * 2.0 ** -24 * (np.abs(k) @ np.abs(q)) + 2.0 ** -25 * np.abs(q).max() * np.abs(k).sum(-1))).max())
    big = p @ np.abs(v)
    tol = 2.0 ** -8 * np.abs(y) + (2 * e + 2.0 ** -20 + len(k) * 2.0 ** -22) * big + (p * weight) @ np.abs(v) + 2.0 ** -134
    return y, lse, tol, e + 2.0 ** -20 + len(k) * 2.0 ** -23 + 2.0 ** -22 * abs(lse)
