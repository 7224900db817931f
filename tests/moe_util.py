"""Inputs and bounds for the tests of the mixture of experts."""
import numpy as np
import torch

from oracle import moe as M
from oracle.quant import e4m3_round

FP = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
Q8 = {"i8": torch.int8, "f8": torch.float8_e4m3fn}
STEP = {"f16": 2.0 ** -11, "bf16": 2.0 ** -8}             # half a step, relative
TINY = {"f16": 2.0 ** -25, "bf16": 2.0 ** -134}           # ... of the subnormals
U = 2.0 ** -24                                            # half a step of FP32


def num(t):
    return t.float().cpu().numpy().astype(np.float64)


def to(x, kind):
    """float64 -> (device tensor of the kind, the numbers that it holds)."""
    if kind == "i8":
        x = np.clip(np.rint(x), -127, 127)
    elif kind == "f8":
        x = e4m3_round(np.clip(x, -448, 448))
    t = torch.from_numpy(np.ascontiguousarray(x, dtype=np.float32)).to(Q8.get(kind) or FP[kind])
    return t.cuda(), num(t)


def f32(x):
    """float64 -> (device FP32 tensor, the same on the host)."""
    x = np.ascontiguousarray(x, dtype=np.float32)
    return torch.from_numpy(x).cuda(), x


def deal(g, counts, T, k_pad=0):
    """A plan with counts[e] rows for expert e: offset, token (device and host) for tokens drawn at random; k_pad more rows that nobody owns."""
    offset = np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    R = int(offset[-1]) + k_pad
    token = g.integers(0, T, max(R, 1)).astype(np.int32)[:R]
    return offset, token, torch.from_numpy(offset).cuda(), torch.from_numpy(token).cuda()


def linear_bounds(y, v, size, act, gated, post, kind, K, offset):
    """How far the device's value before its last rounding may be from y.
    Products: INT8 sums are exact and lose at most half a step as a float; FP sums of K products in an order and with a rounding (truncation at worst) that
    is the tensor core's: (K + 8) 2^-23 of the sum of magnitudes.  Scales and bias: three more roundings.  Activations: GELU(erf) 1.5e-7 absolute
    (its comment), GELU(tanh) tanhf's 2 units and six roundings of x; SiLU: __expf is within 2 + 1.173 |v| units, the quotient within 2 and
    the sum half a unit; slopes at most 1.13."""
    dv = size * ((6 * U) if kind == "i8" else (K + 12) * 2 * U)
    n = v.shape[1] // 2 if gated else v.shape[1]
    g, dg = v[:, :n], dv[:, :n]
    a = M.ACT[act](g)
    da = dg * (1.0 if act == "none" else 1.13)
    if act == "gelu_erf":
        da = da + 1.5e-7
    elif act == "gelu_tanh":
        da = da + 16 * U * np.abs(g)
    elif act == "silu":
        da = da + np.abs(a) * 2 * U * (6 + 1.173 * np.abs(g)) + 2.0 ** -140
    if gated:
        u, du = v[:, n:], dv[:, n:]
        da = da * np.abs(u) + np.abs(a) * du + da * du + 2 * U * np.abs(a * u)
    if post is not None:
        f = np.concatenate([np.repeat(np.abs(np.asarray(post[e], np.float64))[None], offset[e + 1] - offset[e], 0) for e in range(len(offset) - 1)])
        da = da * f
    return da + 3 * U * np.abs(y)


def assert_near(got, want, bar, kind, what=""):
    """got: numbers read back (codes of an 8-bit kind); want: before the last rounding, known to within bar."""
    if kind in ("i8", "f8"):
        d = bar * 1.01 + 1e-30
        assert np.all((got >= M.emit(want - d, kind)) & (got <= M.emit(want + d, kind))), what       # rounding is monotonic
    else:
        assert np.all(np.abs(got - want) <= bar + STEP[kind] * (np.abs(want) + bar) + TINY[kind]), (what, float(np.max(np.abs(got - want))))
