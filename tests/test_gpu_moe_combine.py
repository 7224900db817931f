"""GPU: hero_moe_combine against the oracle."""
import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import hero
from moe_util import FP, Q8, STEP, TINY, U, f32, num, to

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def side(g, rows, H, kind, gran="none", E=None, pad=0):
    """(hero.Tensor, values) of a tensor of the kind; a feature-wise scale is [H], or [E][H] for the experts' rows."""
    t, x = to(g.standard_normal((rows, H)) * {"i8": 36.0, "f8": 60.0}.get(kind, 1.0), kind)
    if pad:
        wide = torch.zeros(rows, H + pad, dtype=t.dtype, device="cuda")
        wide[:, :H].view(torch.int8 if kind in Q8 else t.dtype).copy_(t.view(torch.int8) if kind in Q8 else t)
        t = wide[:, :H]
    if kind not in Q8 or gran == "none":
        return hero.tensor(t), x, None
    s_t, s = f32(np.exp(0.3 * g.standard_normal({"twq": rows, "sq": 1, "fwq": H if E is None else (E, H)}[gran])) / 40)
    return hero.tensor(t, gran, s_t), x, s.astype(np.float64)


def pairs(g, T, k, E, R, drop):
    """Rows without repetition, some places empty."""
    row = g.permutation(max(R, T * k))[:T * k].reshape(T, k) % max(R, 1)
    row[g.random((T, k)) < drop] = -1
    return row.astype(np.int32), g.integers(0, E, (T, k)).astype(np.int32), (g.random((T, k)) + 0.1).astype(np.float32)


def case(h, seed, T, H, k, y="bf16", y_gran="none", res="f16", res_gran="none", shared=None, shared_gran="none", fp="f16", out="i8", out_gran="twq", drop=0.2, pad=0, E=5):
    g = np.random.default_rng(seed)
    R = T * k + 3
    row, expert, weight = pairs(g, T, k, E, R, drop)
    y_t, yv, ys = side(g, R, H, y, y_gran, E, pad)
    t = {n: torch.from_numpy(v).cuda() for n, v in (("row", row), ("expert", expert), ("weight", weight))}
    of = np.zeros(R, int)
    of[row[row >= 0]] = expert[row >= 0]
    yv = yv * (1.0 if ys is None else ys[0] if y_gran == "sq" else ys[of])
    extra = {}
    vals = {}
    for name, kind, gran in (("residual", res, res_gran), ("shared", shared, shared_gran)):
        if kind:
            d, v, s = side(g, T, H, kind, gran, None, pad)
            extra[name], vals[name] = d, v * (1.0 if s is None else s[:, None] if gran == "twq" else s)
    gamma_t, gamma = f32(1 + 0.2 * g.standard_normal(H))
    beta_t, beta = f32(0.1 * g.standard_normal(H))
    fp_t = torch.full((T, H + pad), 3.0, dtype=FP[fp], device="cuda")[:, :H] if fp else None
    o_t = o_s = None
    if out:
        o_t = torch.full((T, H + pad), 3.0, device="cuda").to(Q8.get(out) or FP[out])[:, :H]
        if out in Q8:
            o_s = torch.full({"twq": (T,), "sq": (1,), "fwq": (H,)}[out_gran], 0.03 if out == "i8" else 0.008, device="cuda")
            if out_gran == "fwq":
                o_s.mul_(torch.from_numpy(np.exp(0.3 * g.standard_normal(H)).astype(np.float32)).cuda())
    h.hero_moe_combine(y_t, t["row"], t["weight"], expert=t["expert"] if y_gran == "fwq" else None, out=hero.tensor(o_t, out_gran if out in Q8 else "none", o_s) if out else None,
                       fp_out=hero.tensor(fp_t) if fp else None, gamma=gamma_t if out else None, beta=beta_t if out else None, eps=1e-5, **extra)
    h.check()
    r, size = M.combine(yv, row, weight, **vals)
    # each addend takes three roundings, its sum one for each addend behind it
    bar = (k + 6) * U * size
    if fp:
        got = num(fp_t)
        assert np.all(np.abs(got - r) <= bar + STEP[fp] * (np.abs(r) + bar) + TINY[fp])
        r, bar = got, 0.0                                   # the normalisation reads what is stored
    if not out:
        return
    mean = r.mean(1, keepdims=True)
    std = np.sqrt(r.var(1, keepdims=True) + 1e-5)
    n = (r - mean) / std
    # the mean is off by at most 48 roundings of the mean magnitude (8 to 32 values a thread, 5 shuffles, 16 warps), the centred values by one more,
    # the norm factor relatively by half as many as the variance; gamma, beta and the product three
    dn = (np.broadcast_to(bar, r.shape) + 50 * U * (np.abs(r).mean(1, keepdims=True) + np.abs(r)) + np.broadcast_to(bar, r.shape).max(1, keepdims=True)) / std + 64 * U * np.abs(n)
    want, d = n * gamma + beta, dn * np.abs(gamma) + 3 * U * (np.abs(n * gamma) + np.abs(beta))
    got = num(o_t)
    if out not in Q8:
        assert np.all(np.abs(got - want) <= d + STEP[out] * (np.abs(want) + d) + TINY[out])
        return
    s = num(o_s)
    if out_gran == "twq":
        top = 127 if out == "i8" else 448
        most = np.abs(want).max(1)
        assert np.all(np.abs(s - most / top) <= (d.max(1) + 2 * U * most) / top)
        s = s[:, None]
    q, dq = want / s, d / s + 2 * U * np.abs(want / s)
    assert np.all((got >= M.emit(q - dq, out)) & (got <= M.emit(q + dq, out)))


@pytest.mark.parametrize("T", [1, 5, 70])
@pytest.mark.parametrize("H", [16, 48, 256, 1040, 4096, 4112, 8208, 16384])
@pytest.mark.parametrize("k", [1, 2, 8, 9, 16])
def test_sizes(h, T, H, k):
    if T * H > 70 * 4112:
        T = 7
    case(h, T + H + k, T, H, k)


@pytest.mark.parametrize("T,H,k", [(600, 16, 1), (700, 48, 3), (1000, 1040, 8), (650, 2064, 2), (620, 4096, 8), (601, 4080, 16), (2500, 256, 5)])
@pytest.mark.parametrize("y,y_gran,out,out_gran", [("bf16", "none", "i8", "twq"), ("f16", "none", "f16", "none"), ("i8", "fwq", "i8", "fwq"), ("i8", "sq", "f8", "twq"), ("f8", "fwq", "bf16", "none")])
def test_many_tokens(h, T, H, k, y, y_gran, out, out_gran):
    case(h, T + H, T, H, k, y, y_gran, "f16" if H > 100 else "i8", "none" if H > 100 else "twq", out=out, out_gran=out_gran, drop=0.3, pad=16)


@pytest.mark.parametrize("y,y_gran", [("f16", "none"), ("bf16", "none"), ("i8", "fwq"), ("i8", "sq"), ("i8", "none"), ("f8", "fwq"), ("f8", "sq")])
@pytest.mark.parametrize("res,res_gran", [(None, "none"), ("f16", "none"), ("i8", "twq"), ("i8", "fwq"), ("f8", "twq"), ("bf16", "none")])
def test_operand_types(h, y, y_gran, res, res_gran):
    case(h, 3, 40, 272, 4, y, y_gran, res, res_gran, pad=32)
    case(h, 4, 40, 272, 4, y, y_gran, res, res_gran, shared="i8", shared_gran="sq", fp=None, out="bf16")
    case(h, 5, 40, 272, 4, y, y_gran, res, res_gran, shared="f16", fp="bf16", out=None)


@pytest.mark.parametrize("out,out_gran", [("i8", "twq"), ("i8", "fwq"), ("i8", "sq"), ("f8", "twq"), ("f8", "fwq"), ("f8", "sq"), ("f16", "none"), ("bf16", "none")])
@pytest.mark.parametrize("fp", [None, "f16", "bf16"])
def test_outputs(h, out, out_gran, fp):
    case(h, 6, 33, 528, 3, "i8", "fwq", "i8", "twq", out=out, out_gran=out_gran, fp=fp, pad=16)


def test_tokens_without_a_row_and_dropped_pairs(h):
    case(h, 7, 700, 64, 4, drop=1.0)
    case(h, 8, 700, 64, 4, drop=1.0, res=None, fp=None)
    case(h, 9, 700, 64, 4, drop=0.9, out=None)
    case(h, 7, 50, 64, 4, drop=1.0)                         # the residual alone
    case(h, 8, 50, 64, 4, drop=1.0, res=None, fp=None)      # nothing at all: zeros, scale of beta alone
    case(h, 9, 50, 64, 4, drop=0.7)


def test_a_dropped_pair_adds_nothing_whatever_its_weight(h):
    y = torch.full((4, 32), float("nan"), dtype=torch.bfloat16, device="cuda")
    row, w = torch.full((6, 2), -1, dtype=torch.int32, device="cuda"), torch.full((6, 2), float("inf"), device="cuda")
    fp = torch.full((6, 32), 3.0, dtype=torch.bfloat16, device="cuda")
    h.hero_moe_combine(hero.tensor(y), row, w, fp_out=hero.tensor(fp))
    h.check()
    assert torch.all(fp == 0)


@pytest.mark.parametrize("T", [60, 3000])
def test_an_output_may_be_the_residual(h, T):
    g = np.random.default_rng(10)
    H, k = 512, 3
    row, expert, weight = (torch.from_numpy(x).cuda() for x in pairs(g, T, k, 4, T * k, 0.1))
    y, res = to(g.standard_normal((T * k, H)), "f16")[0], to(g.standard_normal((T, H)), "f16")[0]
    gamma, beta = f32(np.ones(H))[0], f32(np.zeros(H))[0]
    for inplace in (False, True):
        r = res.clone()
        fp = r if inplace else torch.zeros_like(r)
        codes, s = torch.zeros(T, H, dtype=torch.int8, device="cuda"), torch.zeros(T, device="cuda")
        h.hero_moe_combine(hero.tensor(y), row, weight, residual=hero.tensor(r), fp_out=hero.tensor(fp), out=hero.tensor(codes, "twq", s), gamma=gamma, beta=beta)
        h.check()
        if inplace:
            assert torch.equal(fp, first[0]) and torch.equal(codes, first[1]) and torch.equal(s, first[2])      # noqa: F821
        first = (fp, codes, s)


def test_bounds_that_the_host_cannot_see(h):
    y, s = torch.ones(8, 32, dtype=torch.int8, device="cuda"), torch.ones(3, 32, device="cuda")
    w = torch.ones(4, 2, device="cuda")
    i = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda").reshape(4, 2)  # noqa: E731
    fine = (0, 1, 2, 3, 4, 5, 6, 7)
    for row, expert in (((8, 1, 2, 3, 4, 5, 6, 7), (0,) * 8), ((-2, 1, 2, 3, 4, 5, 6, 7), (0,) * 8), (fine, (3,) + (0,) * 7), (fine, (-1,) + (0,) * 7)):
        fp = torch.zeros(4, 32, dtype=torch.float16, device="cuda")
        h.hero_moe_combine(hero.tensor(y, "fwq", s), i(*row), w, expert=i(*expert), fp_out=hero.tensor(fp))
        with pytest.raises(hero.HeroError) as e:
            h.check()
        assert e.value.status == hero.ERR_INVALID_ARG
        assert fp[:, 0].tolist() == [1.0, 2.0, 2.0, 2.0]
    h.check()


def test_refusals_of_the_binding(h):
    y, fp = torch.zeros(8, 32, dtype=torch.int8, device="cuda"), torch.zeros(4, 32, dtype=torch.float16, device="cuda")
    row, w, s = torch.zeros(4, 2, dtype=torch.int32, device="cuda"), torch.zeros(4, 2, device="cuda"), torch.ones(3, 32, device="cuda")
    good = dict(y=hero.tensor(y, "fwq", s), row=row, weight=w, expert=row, fp_out=hero.tensor(fp))
    for bad in (dict(y=hero.tensor(y, "fwq", s[0])), dict(row=row[:3]), dict(row=row.long()), dict(weight=w[:, :1]), dict(expert=None), dict(expert=row[:, :1]),
                dict(fp_out=None), dict(out=hero.tensor(y[:4], "twq", s[0, :4].contiguous())), dict(residual=hero.tensor(y[:4], "twq", s[0, :3].contiguous())),
                dict(out=hero.tensor(y[:4], "fwq", s[0, :16].contiguous()), gamma=s[0], beta=s[0])):
        with pytest.raises(hero.HeroError):
            h.hero_moe_combine(**dict(good, **bad))
    h.check()
