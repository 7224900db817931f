"""A mixture of experts: the router's choice and order, the experts' products, the weighted sum with LN^quant (oracle; test
infrastructure only).  fp64 throughout, plain loops."""
import numpy as np

from . import ops as O
from .quant import F8MAX, QMAX, e4m3_round


def scores(x, score):
    """[T, E] logits -> scores; -inf and NaN take no part (score 0); several +inf share a softmax equally."""
    x = np.asarray(x, np.float64)
    part = x > -np.inf                                     # (False for NaN)
    if score == "sigmoid":
        with np.errstate(over="ignore"):
            return np.where(part, 1 / (1 + np.exp(-np.where(part, x, 0.0))), 0.0)
    out = np.zeros_like(x)
    for t in range(x.shape[0]):
        if part[t].any():
            m = x[t][part[t]].max()
            with np.errstate(invalid="ignore"):
                e = np.where(part[t], np.where(x[t] == m, 1.0, np.exp(x[t] - m)), 0.0)
            out[t] = e / e.sum()
    return out


def route(x, k, score="softmax", renorm=True, scale=1.0, bias=None, n_tokens=None):
    """Returns expert, weight [T, k], offset [E + 1], token (sorted rows in use), row [T, k]."""
    x = np.array(x, np.float64)
    T, E = x.shape
    if bias is not None:
        b = np.asarray(bias, np.float64)
        x[:, ~(b > -np.inf)] = -np.inf
    part = x > -np.inf
    s = scores(x, score)
    key = x if bias is None else s + np.where(b > -np.inf, b, 0.0)
    expert, weight = np.full((T, k), -1, np.int64), np.zeros((T, k))
    for t in range(T if n_tokens is None else min(max(n_tokens, 0), T)):
        order = sorted((e for e in range(E) if part[t, e]), key=lambda e: (-key[t, e], e))[:k]
        if not order:
            continue
        w = s[t, order]
        if renorm:
            # in logarithms, so that scores too small for a double keep their ratios
            z = x[t, order]
            with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
                g = np.minimum(z, 0) - np.log1p(np.exp(-np.abs(z))) if score == "sigmoid" else z
                w = np.where(g == g.max(), 1.0, np.exp(g - g.max()))
            w = w / w.sum()
        expert[t, :len(order)], weight[t, :len(order)] = order, w * scale
    offset, token, row = [0], [], np.full((T, k), -1, np.int64)
    for e in range(E):
        for t in range(T):
            for j in range(k):
                if expert[t, j] == e:
                    row[t, j] = len(token)
                    token.append(t)
        offset.append(len(token))
    return expert, weight, np.array(offset), np.array(token, np.int64), row


def silu(v):
    with np.errstate(over="ignore"):
        return v / (1 + np.exp(-v))


ACT = {"none": lambda v: v, "gelu_erf": O.gelu_erf, "gelu_tanh": O.gelu_tanh, "silu": silu}


def linear(a, rs, W, cs, bias, act, gated, post, offset, token):
    """The sorted rows' products before rounding, [offset[-1], columns], and two sizes that error bounds are made of: sum_c |a w| (with scales,
    plus |bias|), of the gate (or only) half and of the other half.  a [rows, K], W [E, N, K], both as numbers."""
    a, W = np.asarray(a, np.float64), np.asarray(W, np.float64)
    n_out = W.shape[1] // 2 if gated else W.shape[1]
    y, v_all, size = (np.zeros((offset[-1], c)) for c in (n_out, W.shape[1], W.shape[1]))
    for e in range(W.shape[0]):
        for r in range(offset[e], offset[e + 1]):
            i = r if token is None else token[r]
            f = 1.0 if rs is None else np.float64(rs[i])
            c = 1.0 if cs is None else np.asarray(cs[e], np.float64)
            b = 0.0 if bias is None else np.asarray(bias[e], np.float64)
            v = W[e] @ a[i] * f * c + b
            v_all[r], size[r] = v, np.abs(W[e]) @ np.abs(a[i]) * f * np.abs(c) + np.abs(b)
            g = ACT[act](v[:n_out]) * v[n_out:] if gated else ACT[act](v)
            y[r] = g if post is None else g * np.asarray(post[e], np.float64)
    return y, v_all, size


def emit(y, kind):
    """Values -> what an output of that kind holds, before the 16-bit types' rounding: codes of I8 / F8."""
    if kind == "i8":
        return np.clip(np.rint(y), -QMAX, QMAX)
    return e4m3_round(np.clip(y, -F8MAX, F8MAX)) if kind == "f8" else y


def combine(y, row, weight, residual=None, shared=None):
    """Sums r [T, H] and sum of magnitudes; y, residual, shared as values (dequantised)."""
    T, H = row.shape[0], y.shape[1]
    r, size = np.zeros((T, H)), np.zeros((T, H))
    for t in range(T):
        for x in (residual, shared):
            if x is not None:
                r[t] += x[t]
                size[t] += np.abs(x[t])
        for j in range(row.shape[1]):
            if row[t, j] >= 0:
                r[t] += np.float64(weight[t, j]) * y[row[t, j]]
                size[t] += np.abs(np.float64(weight[t, j]) * y[row[t, j]])
    return r, size
