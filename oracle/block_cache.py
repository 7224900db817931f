"""The 8-bit block cache, the attention over it, and the norm and rotation of query / key heads (oracle; test
infrastructure only).  fp64, except where the definition itself is in FP32: the codes of the append are the FP32 quotient
x / s rounded, so numpy's float32 (correctly rounded) division states them to the bit."""
import numpy as np

from .quant import F8MAX, QMAX, e4m3_round


def top(kind):
    return float(QMAX if kind == "i8" else F8MAX)


def to_codes(y, kind):
    """FP32 quotients -> code values (fp64): clip(RNE) or saturating e4m3; NaN -> 0."""
    y = np.where(np.isnan(y), 0.0, np.asarray(y, np.float64))
    y = np.clip(y, -top(kind), top(kind))
    return np.rint(y) if kind == "i8" else e4m3_round(y)


def divide(x, s):
    """FP32 division by a scale; everything is 0 under a zero scale."""
    x, s = np.asarray(x, np.float32), np.float32(s)
    if s == 0:
        return np.zeros_like(x)
    with np.errstate(over="ignore", invalid="ignore"):
        return x / s


def append(codes, scale, table, lens, counts, starts, x, page, kind):
    """codes [pages, heads, page, dh] (values, fp64) and scale [pages, heads] (FP32) after the last counts[b] tokens of each
    sequence, rows starts[b].. of x [rows, heads * dh], have been stored.  Returns new arrays."""
    codes, scale = codes.copy(), np.asarray(scale, np.float32).copy()
    _, heads, _, dh = codes.shape
    for b, n in enumerate(counts):
        begin = lens[b] - n
        first = max(begin, 0)
        for pi in range(first // page, -(-lens[b] // page) if lens[b] > first else 0):
            p0, pid = pi * page, table[b][pi]
            if not 0 <= pid < codes.shape[0]:
                continue
            lo, hi = max(first - p0, 0), min(lens[b] - p0, page)
            new = np.asarray(x[starts[b] + p0 + lo - begin:starts[b] + p0 + hi - begin], np.float32).reshape(hi - lo, heads, dh)
            for g in range(heads):
                fin = np.abs(new[:, g][np.isfinite(new[:, g])])
                amax = np.float32(fin.max()) if fin.size else np.float32(0)
                s_old = scale[pid, g] if lo > 0 else np.float32(0)
                s = max(s_old, amax / np.float32(top(kind)))
                if lo > 0 and s > s_old:
                    codes[pid, g, :lo] = to_codes(divide(codes[pid, g, :lo].astype(np.float32) * s_old, s), kind)
                codes[pid, g, lo:hi] = to_codes(divide(new[:, g], s), kind)
                scale[pid, g] = s
    return codes, scale


def tokens(codes, scale, table_row, n, page):
    """Values of a sequence's first n tokens, [n, heads, dh]; page ids are clamped into the pool."""
    ids = np.clip(np.asarray(table_row[:max(1, -(-n // page))]), 0, codes.shape[0] - 1)
    y = codes[ids] * np.asarray(scale, np.float64)[ids][:, :, None, None]
    return y.transpose(0, 2, 1, 3).reshape(-1, codes.shape[1], codes.shape[3])[:n]


def attention(q, k, v, group, scale):
    """Rows q [n, nq, dh] are the last n of the tokens k, v [L, nkv, dh]; causal.  Returns (o [n, nq, dh], sum_k P |v|,
    largest sum_c |q_c k_c| scale over the keys of a row [n, nq]): the last two are what error bounds are made of."""
    n, nq, dh = q.shape
    L = k.shape[0]
    o, mass, size = np.zeros((n, nq, dh)), np.zeros((n, nq, dh)), np.zeros((n, nq))
    for i in range(n):
        m = L - n + i + 1
        if m <= 0:
            continue
        for j in range(nq):
            kk, vv = k[:m, j // group], v[:m, j // group]
            s = kk @ q[i, j] * scale
            p = np.exp(s - s.max())
            p /= p.sum()
            o[i, j], mass[i, j] = p @ vv, p @ np.abs(vv)
            size[i, j] = (np.abs(kk) @ np.abs(q[i, j])).max() * abs(scale)
    return o, mass, size


def norm_rope(x, heads, gamma, eps, cos, sin, pos, pairing):
    """x [rows, heads * dh] -> the same shape, fp64.  gamma None: no norm; cos None: no rotation."""
    rows = x.shape[0]
    y = np.asarray(x, np.float64).reshape(rows, heads, -1)
    if gamma is not None:
        y = y / np.sqrt((y * y).mean(-1, keepdims=True) + eps) * np.asarray(gamma, np.float64)
    if cos is not None:
        half = cos.shape[1]
        a = np.arange(half) if pairing == "halves" else np.arange(0, 2 * half, 2)
        b = a + (half if pairing == "halves" else 1)
        pos = np.clip(np.asarray(pos), 0, cos.shape[0] - 1)
        c, s = (np.asarray(t, np.float64)[pos][:, None] for t in (cos, sin))
        z = y.copy()
        z[..., a] = y[..., a] * c - y[..., b] * s
        z[..., b] = y[..., b] * c + y[..., a] * s
        y = z
    return y.reshape(rows, -1)
