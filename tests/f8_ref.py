"""64-bit statements of the 8-bit floating point layers and of the operators on logits, for the tests (numpy only)."""
import numpy as np

FMAX = {"e4m3": 448.0, "e5m2": 57344.0}


def decode(codes, fmt):
    """Values of e4m3 / e5m2 codes (uint8)."""
    c = np.arange(256)
    sign = np.where(c & 128, -1.0, 1.0)
    if fmt == "e4m3":
        e, m = (c >> 3) & 15, c & 7
        v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (e - 10.0))
        v = np.where((c & 127) == 127, np.nan, v)
    else:
        e, m = (c >> 2) & 31, c & 3
        v = np.where(e == 0, m * 2.0 ** -16, (4 + m) * 2.0 ** (e - 17.0))
        v = np.where(e == 31, np.where(m == 0, np.inf, np.nan), v)
    return (sign * v)[codes]


def scale_for(amax, fmt):
    """The least power of two (2^-126 at least) with which amax fits."""
    e = -126
    if amax > 0:
        m, x = np.frexp(np.float64(amax) / FMAX[fmt])  # m in [0.5, 1): amax / FMAX = m 2^x
        e = max(e, int(x) - 1 if m == 0.5 else int(x))
    return 2.0 ** e


def nearest(v, fmt):
    """v rounded to the format, ties to even (|v| at most the largest code)."""
    bits, least = (3, -6) if fmt == "e4m3" else (2, -14)
    _, e = np.frexp(v)
    step = 2.0 ** (np.maximum(e - 1, least) - bits)
    return np.rint(v / step) * step


def quantize(x, fmt, block_rows):
    """(values, scales [blocks of columns][rows or blocks of rows]) of x [R][C] in 64 bits."""
    x = np.asarray(x, dtype=np.float64)
    R, C = x.shape
    rb, cb = -(-R // block_rows), -(-C // 128)
    fine = np.isfinite(x)
    a = np.zeros((rb * block_rows, cb * 128))
    a[:R, :C] = np.where(fine, np.abs(x), 0)
    amax = a.reshape(rb, block_rows, cb, 128).max(axis=(1, 3))
    s = np.vectorize(lambda v: scale_for(v, fmt))(amax)
    each = np.repeat(np.repeat(s, block_rows, 0)[:R], 128, 1)[:, :C]
    with np.errstate(invalid="ignore"):
        v = np.where(fine, nearest(np.where(fine, x, 0) / each, fmt), np.nan)
    return v, s.T.copy()


def hswish(y):
    return y * np.clip(y + 3, 0, 6) / 6


def linear(xv, sx, wv, sw, w_block, bias, act, M, K, C):
    """(y, sum of magnitudes) of the layer on code values xv [M][C], wv [>= K][>= C] and scales, 64 bits."""
    cb = -(-C // 128)
    block = np.arange(C) // 128
    x = xv[:M, :C] * sx[:cb, :M].astype(np.float64).T[:, block]
    w = wv[:K, :C] * sw[:cb][:, np.arange(K) // w_block].astype(np.float64).T[:, block]
    y, size = x @ w.T, np.abs(x) @ np.abs(w).T
    if bias is not None:
        y = y + bias[:K]
        size = size + np.abs(bias[:K])
    if act == 1:
        y = np.maximum(y, 0)
    elif act == 2:
        y = hswish(y)
    return y, size


def linear_tolerance(y, size, C, act, bf16):
    """A block's 128 exact products and the block sums are added in fp32, in any order, the tensor core's additions cut off rather than
    rounded (2^-23 of the magnitudes each): 128 + blocks + 4 additions.  h-swish has slope 1.5 at most and three roundings of its own;
    bf16 rounds once more, half a step."""
    t = (128 + -(-C // 128) + 4) * 2.0 ** -23 * size
    if act == 2:
        t = 1.5 * t + 4 * 2.0 ** -24 * np.abs(y)
    if bf16:
        t = t + 2.0 ** -8 * (np.abs(y) + t)
    return t + 1e-30


def top(z, k):
    """Indices of the k largest of every row: largest first, NaN above all, equal values (and zeros) by index."""
    z = np.asarray(z, dtype=np.float64) + 0.0
    z = np.where(np.isnan(z), np.inf, z), np.isnan(z)
    return np.stack([np.lexsort((np.arange(r.size), -r, ~n))[:k] for r, n in zip(*z)])


def distill(z, teacher, index, T, coef):
    """Loss, statistics, gradient, student's q and teacher's total probability of each class, 64 bits; coef [rows]: grad_scale * row_scale."""
    z = np.asarray(z, dtype=np.float64)
    M, V = z.shape
    loss, stat, dz, Q, P = np.zeros(M), np.zeros((M, 2)), np.zeros((M, V)), np.zeros((M, V)), np.zeros((M, V))
    for r in range(M):
        top = z[r].max()
        base = 0.0 if top == -np.inf else top
        with np.errstate(divide="ignore"):
            logsum = np.log(np.exp((z[r] - base) / T).sum())
        stat[r] = top, logsum
        log_q = (z[r] - base) / T - (0.0 if top == -np.inf else logsum)
        Q[r] = np.exp(log_q)
        use = (index[r] >= 0) & (index[r] < V) & (teacher[r] > -np.inf)
        if not use.any():
            continue
        t = teacher[r][use].astype(np.float64) / T
        log_p = t - t.max() - np.log(np.exp(t - t.max()).sum())
        p = np.exp(log_p)
        loss[r] = T * T * np.sum(np.where(p > 0, p * (log_p - log_q[index[r][use]]), 0))
        np.add.at(P[r], index[r][use], p)
        dz[r] = coef[r] * T * (Q[r] - P[r])
    return loss, stat, dz, Q, P


def distill_size(z, teacher, index, T):
    """Largest exponent in use, per row: |z - max| / T over named classes, |log sum|, |teacher - max| / T."""
    z = np.asarray(z, dtype=np.float64)
    out = np.zeros(z.shape[0])
    for r in range(z.shape[0]):
        use = (index[r] >= 0) & (index[r] < z.shape[1]) & (teacher[r] > -np.inf)
        named = z[r][index[r][use]]
        named = named[np.isfinite(named)]
        top = z[r].max()
        if not use.any() or top == -np.inf:
            continue
        out[r] = (np.max(top - named, initial=0) + np.ptp(teacher[r][use].astype(np.float64))) / T + np.log(z.shape[1])
    return out


def distill_tolerance(z, teacher, index, T):
    """Roundings of a row, relative to the terms they belong to: an exponent (difference, product with 1 / T and log2 e: four roundings
    of its own size A), exp and log (two steps each), sums over V / 512 terms a thread and a tree, over the slots likewise."""
    A = distill_size(z, teacher, index, T)
    return 2.0 ** -24 * (64 + z.shape[1] / 256 + 8 * A) * (1 + A)
