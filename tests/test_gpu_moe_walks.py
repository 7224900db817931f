"""GPU: hero_moe_linear where a CTA or a pair of them walks over many ragged tiles (several rounds, a last one that is cut, experts without rows between them), against the
definition in 64 bits, with every factor that the epilogue applies; and an expert's output factors taken from the observer."""
import math

import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import hero
from moe_util import FP, Q8, STEP, TINY, U, deal, f32, num, to

pytestmark = pytest.mark.gpu
SPREAD = {"i8": 36.0, "f8": 60.0, "bf16": 1.0, "f16": 1.0}


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def activate(v, dv, act):
    """Activation of v, known to within dv, in 64 bits, and how far the kernel's may be.  Slopes are at most 1.13.  GELU(erf): 1.5e-7.  SiLU and GELU(tanh) are v / (1 + 2^x): the
    exponent's roundings (1.5 and 4.5 units of 2^-24 of x, 8 units for a sum with 15) reach the power times ln 2, which adds 2^-22 of its own; four
    more for the sum, the reciprocal and the product."""
    if act == "none":
        return v, dv
    if act == "gelu_erf":
        return 0.5 * v * torch.special.erfc(-v / math.sqrt(2)), 1.13 * dv + 1.5e-7
    x = -v / math.log(2) if act == "silu" else -2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3) / math.log(2)
    a = v / (1 + torch.exp2(x))
    return a, 1.13 * dv + U * (0.7 * (8 + (1.5 if act == "silu" else 4.5) * x.abs()) + 8) * a.abs() + 2.0 ** -134


def expert_rows(a, rs, w, cs, b, act, gated, post, kind):
    """One expert's rows before their last rounding, and how far the kernel's may be: INT8 sums are exact and lose half a step as a float, sums of K floating-point products
    lose (K + 8) 2^-23 of the sum of magnitudes whatever their order; scales and bias three more roundings."""
    K = a.shape[1]
    f = (1.0 if rs is None else rs[:, None]) * (1.0 if cs is None else cs[None])
    v = a @ w.T * f + (0.0 if b is None else b)
    size = a.abs() @ w.abs().T * f + (0.0 if b is None else b.abs())
    dv = size * (6 * U if kind == "i8" else (K + 12) * 2 * U)
    n = v.shape[1] // 2 if gated else v.shape[1]
    y, dy = activate(v[:, :n], dv[:, :n], act)
    if gated:
        u, du = v[:, n:], dv[:, n:]
        y, dy = y * u, dy * u.abs() + y.abs() * du + dy * du + 2 * U * (y * u).abs()
    if post is not None:
        y, dy = y * post, dy * post.abs()
    return y, dy + 3 * U * y.abs()


def near(got, want, bar, kind):
    if kind == "i8":
        return bool(((got >= (want - bar).round().clamp(-127, 127)) & (got <= (want + bar).round().clamp(-127, 127))).all())
    if kind == "f8":
        want, bar, got = (t.cpu().numpy() for t in (want, bar, got))
        return bool(np.all((got >= M.emit(want - bar, "f8")) & (got <= M.emit(want + bar, "f8"))))
    return bool(((got - want).abs() <= bar + STEP[kind] * (want.abs() + bar) + TINY[kind]).all())


@pytest.mark.parametrize("top", [600, 40])                # pairs of CTAs, about 200 pieces on 74; single CTAs, more than 1000 on 296
@pytest.mark.parametrize("gather", [True, False])
@pytest.mark.parametrize("kind,out,act,gated,K,N", [("i8", "i8", "silu", True, 1040, 1024), ("i8", "f16", "none", False, 528, 2064), ("i8", "bf16", "gelu_erf", False, 272, 1040),
                                                    ("f8", "bf16", "silu", True, 1040, 544), ("f8", "f8", "gelu_tanh", False, 400, 784), ("bf16", "bf16", "gelu_tanh", False, 520, 1040),
                                                    ("f16", "i8", "gelu_tanh", True, 264, 1120)])
def test_many_ragged_tiles(h, top, gather, kind, out, act, gated, K, N):
    g = np.random.default_rng(top + K)
    E, T, q8 = 64, 500, kind in Q8
    counts = g.integers(0, top, E) * (g.random(E) < 0.8)
    counts[:3] = 1, 257, 5
    offset, token, offset_t, token_t = deal(g, counts, T, 6)
    R, n_out = len(token), N // 2 if gated else N
    at, _ = to(g.standard_normal((T if gather else R, K)) * SPREAD[kind], kind)
    wt, _ = to(g.standard_normal((E, N, K)) * SPREAD[kind] / (1 if q8 else np.sqrt(K)), kind)
    rs = f32(np.exp(0.3 * g.standard_normal(at.shape[0])) / SPREAD[kind])[0] if q8 else None
    cs = f32(np.exp(0.3 * g.standard_normal((E, N))) / (SPREAD[kind] * np.sqrt(K)))[0] if q8 else None
    b = f32(0.5 * g.standard_normal((E, N)))[0]
    post = f32({"i8": 40.0, "f8": 60.0}.get(out, 1.0) * np.exp(0.3 * g.standard_normal((E, n_out))))[0]
    y = torch.full((R, n_out), 3.0, device="cuda").to(Q8.get(out) or FP[out])
    h.hero_moe_linear(hero.tensor(at, "twq", rs) if q8 else hero.tensor(at), wt, hero.tensor(y), offset_t, token=token_t if gather else None, w_scale=cs, bias=b, act=act, gated=gated,
                      post_scale=post)
    h.check()
    d = lambda t: None if t is None else t.float().double()  # noqa: E731
    for e in range(E):
        r = slice(int(offset[e]), int(offset[e + 1]))
        if r.start == r.stop:
            continue
        i = token_t[r].long() if gather else torch.arange(r.start, r.stop, device="cuda")
        want, bar = expert_rows(d(at)[i], d(rs)[i] if q8 else None, d(wt[e]), d(cs[e]) if q8 else None, d(b[e]), act, gated, d(post[e]), kind)
        assert near(d(y[r]), want, bar, out), e
    assert bool((d(y[int(offset[-1]):]) == 3).all())


@pytest.mark.parametrize("top", [300, 20])
@pytest.mark.parametrize("gated", [True, False])
def test_output_factors_from_the_observer_use_the_codes_whole_range(h, top, gated):
    # a batch in 16 bits gives each expert's column maxima, from which the static scales of its hidden features are taken
    g = np.random.default_rng(top)
    E, T, K, N = 40, 300, 256, 320
    counts = g.integers(0, top, E)
    counts[[3, 17]] = 0
    offset, token, offset_t, token_t = deal(g, counts, T)
    n_out = N // 2 if gated else N
    at, wt, b = to(g.standard_normal((T, K)), "f16")[0], to(g.standard_normal((E, N, K)) / 16, "f16")[0], f32(0.3 * g.standard_normal((E, N)))[0]
    fp, codes, most = torch.zeros(len(token), n_out, dtype=torch.float16, device="cuda"), torch.zeros(len(token), n_out, dtype=torch.int8, device="cuda"), torch.zeros(E, n_out, device="cuda")
    call = lambda out, **kw: h.hero_moe_linear(hero.tensor(at), wt, hero.tensor(out), offset_t, token=token_t, bias=b, act="silu", gated=gated, **kw)  # noqa: E731
    call(fp, out_col_absmax=most)
    post = torch.where(most > 0, 127 / most, 1.0)
    call(codes, post_scale=post)
    h.check()
    fp, codes, post = num(fp), num(codes), num(post)
    for e in range(E):
        r = slice(offset[e], offset[e + 1])
        if r.start == r.stop:
            assert not bool(most[e].any())
            continue
        assert np.all(np.abs(codes[r]).max(0) == 127)      # (127 times at most 1 + 2^-11 and a few units)
        # the two calls' values are the same but for the stored one's rounding, half a step of FP16 (or of its subnormals), and three of FP32
        assert np.all(np.abs(codes[r] - fp[r] * post[e]) <= 0.5 + (np.abs(fp[r]) * (2.0 ** -11 + 2.0 ** -21) + 2.0 ** -25) * post[e])
