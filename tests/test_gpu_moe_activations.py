"""GPU: the activations of hero_moe_linear over all that the output types hold, down to results that are subnormal in BF16.  The operands are zero, so that
the bias alone is what the activation gets, exactly."""
import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import hero
from moe_util import FP, STEP, TINY, U, f32, num

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def definition(v, act):
    """In 64 bits, and how far FP32 arithmetic may be from it.  Both are v / (1 + 2^x).  The exponent: SiLU one constant and one rounding (1.5 units of 2^-24 of x), GELU(tanh)
    two constants and three (4.5); both a sum with 15, which rounds by at most 2^-21 up to x = 31 and 2^-24 x beyond, counted above.  2^x: 2^-22
    (ex2.approx's bound), so the power is off by ln 2 (8 + 1.5 |x|) + 4 units, and the quotient by that, one for the sum, two for
    rcp.approx (one in the last place), one for the product with v.  The reciprocal may be subnormal: 2^-150 of v, and as much for the result."""
    v = np.asarray(v, np.float64)
    x = -v / np.log(2.0) if act == "silu" else -2 * np.sqrt(2 / np.pi) * (v + 0.044715 * v ** 3) / np.log(2.0)
    with np.errstate(over="ignore"):
        a = v / (1 + np.exp2(x))
    units = 0.7 * (8 + (1.5 if act == "silu" else 4.5) * np.abs(x)) + 4 + 4
    return a, np.minimum(units * U, 1) * np.abs(a) + 2.0 ** -150 * (np.abs(v) + 1)


def values(act):
    low, far = (-110, -93) if act == "silu" else (-11.5, -10)
    v = np.concatenate([np.linspace(low, 20, 3000), np.linspace(low, 0.8 * far, 1500), [0, -0.0, -88, -10.05, -87.34, -88.73, 1e-30, -1e-30, 1e-42, 300, 1e15, -200, -1e15],
                        np.logspace(-36, 0, 90), -np.logspace(-36, 0, 89)])
    return np.resize(v, 4704).astype(np.float32)


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("rows", [3, 70])                 # both forms of the kernel
@pytest.mark.parametrize("kind,out", [("bf16", "bf16"), ("i8", "bf16"), ("i8", "f16"), ("f16", "f16"), ("i8", "i8")])
def test_small_results(h, act, gated, rows, kind, out):
    v = values(act)
    n, K = len(v), 32
    N = 2 * n if gated else n
    up = np.resize(np.float32([1, -1, 0.75, 3]), n)
    b_t, _ = f32(np.concatenate([v, up])[None] if gated else v[None])
    dt = {"i8": torch.int8}.get(kind) or FP[kind]
    a, w = torch.zeros(rows, K, dtype=dt, device="cuda"), torch.zeros(1, N, K, dtype=dt, device="cuda")
    y = torch.full((rows, n), 3, device="cuda").to({"i8": torch.int8}.get(out) or FP[out])
    # codes: an output factor that brings the smallest of the results back
    post = 2.0 ** 122 if out == "i8" else 1.0
    h.hero_moe_linear(hero.tensor(a), w, hero.tensor(y), torch.tensor([0, rows], dtype=torch.int32, device="cuda"), w_scale=torch.ones(1, N, device="cuda") if kind == "i8" else None,
                      bias=b_t, act=act, gated=gated, post_scale=torch.full((1, n), post, device="cuda") if out == "i8" else None)
    h.check()
    want, bar = definition(v, act)
    if gated:
        want, bar = want * up, bar * np.abs(up) + U * np.abs(want * up) + 2.0 ** -150
    want, bar = want * post, bar * post * 1.01 + U * np.abs(want * post)
    # a reciprocal below the normal range is 0: from x = 141 on, where the result is below 2^-134.3
    bar = bar + np.where(np.abs(want) < 3 * 2.0 ** -134.3 * post, np.abs(want), 0)
    got = num(y)
    assert np.all(got == got[0])
    if out == "i8":
        with np.errstate(over="ignore"):
            assert np.all((got[0] >= M.emit(want - bar, out)) & (got[0] <= M.emit(want + bar, out)))
        return
    fits = np.abs(want) < (6e4 if out == "f16" else 3e38)
    assert np.all((np.abs(got[0] - want) <= bar + STEP[out] * (np.abs(want) + bar) + TINY[out])[fits])
