"""Plain 64-bit forms of the 8-bit caches, of attention with its weights and of
eviction, written from their definitions (include/catekv_cache.h), on numpy."""
import math

import numpy as np

D = 128


def bf16_round(x):
    """fp64 or fp32 -> the nearest bf16 (ties to even), as fp32."""
    b = np.asarray(x, dtype=np.float32).view(np.uint32).astype(np.uint64)
    r = ((b + 0x7FFF + ((b >> 16) & 1)) >> 16 << 16).astype(np.uint32).view(np.float32)
    return np.where(np.isnan(x), np.float32(np.nan), r)


# every finite e4m3 value, by code 0 .. 126
E4M3 = np.array([m * 2.0 ** -9 for m in range(8)] +
                [(8 + m) * 2.0 ** (e - 10) for e in range(1, 16) for m in range(8)][:119])


def e4m3_value(codes):
    c = np.asarray(codes, dtype=np.uint8)
    v = np.concatenate([E4M3, [np.nan]])[c & 127]
    return np.where(c & 128, -v, v)


def block_scale(x, fmt):
    """Scale (fp32) of one block, NaN for a block that is not finite."""
    if not np.isfinite(x).all():
        return np.float32(np.nan)
    m = np.abs(x).max()
    if m < 2.0 ** -100:
        return np.float32(0)
    if fmt == "int8":
        return np.float32(np.float32(m) * np.float32(1.0 / 127.0))
    e = math.frexp(m)[1] - 9                       # m <= 2^(e + 9): 448 2^e or 448 2^(e + 1) suffices
    return np.float32(2.0 ** (e if m <= 448 * 2.0 ** e else e + 1))


def block_codes(x, fmt, scale):
    """Codes [..] uint8 of one block (fp64 rows x)."""
    if not scale > 0:
        return np.zeros(x.shape, dtype=np.uint8)
    y = x.astype(np.float64) / np.float64(scale)
    if fmt == "int8":
        return np.clip(np.rint(y), -127, 127).astype(np.int8).view(np.uint8)
    a = np.abs(y)
    hi = np.clip(np.searchsorted(E4M3, a), 1, len(E4M3) - 1)
    lo = hi - 1
    down, up = a - E4M3[lo], E4M3[hi] - a
    code = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo).astype(np.uint8)
    return code | np.where(np.signbit(x), 128, 0).astype(np.uint8)


def quantize(rows, fmt, block):
    """rows [L][D] (fp64 of stored values) -> (codes [nb block][D] uint8, scales [nb] fp32)."""
    nb = len(rows) // block
    codes, scales = np.zeros((nb * block, D), dtype=np.uint8), np.zeros(nb, dtype=np.float32)
    for b in range(nb):
        x = rows[b * block:(b + 1) * block]
        scales[b] = block_scale(x, fmt)
        codes[b * block:(b + 1) * block] = block_codes(x, fmt, scales[b])
    return codes, scales


def values(codes, scales, fmt, block):
    """fp64 values of codes, exactly."""
    v = codes.view(np.int8).astype(np.float64) if fmt == "int8" else e4m3_value(codes)
    return v * np.repeat(scales.astype(np.float64), block)[:, None]


def attend(q, k, v, scale):
    """q [G][D] over rows k, v: (out [G][D], lse [G], mean weight per row,
    largest sum |q||k| scale, sum p |v| [G][D])."""
    if not len(k):
        return np.zeros((len(q), D)), np.full(len(q), -np.inf), np.zeros(0), 0.0, np.zeros((len(q), D))
    s = q @ k.T * scale
    m = s.max(axis=1, keepdims=True)
    p = np.exp(s - m)
    l = p.sum(axis=1, keepdims=True)
    p /= l
    return (p @ v, (m + np.log(l))[:, 0], p.mean(axis=0), float((np.abs(q) @ np.abs(k).T).max() * scale),
            p @ np.abs(v))


def score_error(sum_abs):
    """Largest error of a score whose products' magnitudes sum to sum_abs: at most
    128 fp32 additions, each off by 2^-24 of at most that sum, and six more
    roundings of the score (the scales, the factor and the subtraction of the
    maximum), which is no larger; a query in two fp16 parts or a power-of-two
    scaled one is off by at most 2^-22."""
    return sum_abs * ((128 + 6) * 2.0 ** -24 + 2.0 ** -22)


def weight_error(sum_abs, rows):
    """Relative error of a softmax weight: e^(2 d) - 1 for scores off by d, with
    exp2 and its argument's rounding (3 2^-23) and sums of fp32 over the rows,
    which a tree of at most 64 sequential additions per lane and segment and
    rows / 64 / 8 of them bounds."""
    d = score_error(sum_abs)
    return math.expm1(2 * d) + (6 + min(rows, 64 + rows / 512)) * 2.0 ** -23


def output_error(sum_abs, rows):
    """Error of an output over sum p |v|: the weight's, P's split (2^-21), and as
    many additions again."""
    return weight_error(sum_abs, rows) + 2.0 ** -21 + (64 + rows / 64) * 2.0 ** -24


def weight_order(acc):
    """acc as a sortable float64: NaN above everything."""
    a = np.asarray(acc, dtype=np.float64)
    return np.where(np.isnan(a), np.inf, a), np.isnan(a)


def evict(acc, budget, cs, recent):
    """Source row of every remaining row of one view with len(acc) rows."""
    L = len(acc)
    nc = max(L - recent, 0) // cs
    if budget < 0 or nc <= budget:
        return np.arange(L)
    k = budget
    best = []
    for c in range(nc):
        a = acc[c * cs:(c + 1) * cs]
        best.append((1, 0.0) if np.isnan(a).any() else (0, float(a.max())))
    order = sorted(range(nc), key=lambda c: (-best[c][0], -best[c][1], c))
    stay = sorted(order[:k])
    place = list(range(k))
    movers = [c for c in stay if c >= k]
    for hole in [c for c in range(k) if c not in set(stay)]:
        place[hole] = movers.pop(0)
    rows = [c * cs + i for c in place for i in range(cs)]
    return np.array(rows + list(range(nc * cs, L)), dtype=np.int64)
