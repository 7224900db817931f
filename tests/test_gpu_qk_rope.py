"""GPU parity: hero_qk_norm_rope against the oracle in fp64.  Bounds: the norm factor and every product are FP32 (a few units of
2^-24, counted as 16), the result is rounded once to its type (half a step); a rotated feature is a sum of two products,
so the FP32 part is relative to |a cos| + |b sin|."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero
from block_util import FP, to_fp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def _tables(n, rot, seed=0):
    th = np.arange(n)[:, None] * 10000.0 ** (-np.arange(rot // 2) / (rot // 2)) + seed
    c, s = np.cos(th).astype(np.float32), np.sin(th).astype(np.float32)
    return c, s, torch.from_numpy(c).cuda(), torch.from_numpy(s).cuda()


def _bound(x, heads, gamma, eps, cos, sin, pos, pairing, fp):
    """Half a step of the type on the value, 16 units of 2^-24 on the sum of magnitudes."""
    mag = BC.norm_rope(np.abs(x), heads, None if gamma is None else np.abs(gamma), eps, None, None, None, pairing) if cos is None else None
    y = BC.norm_rope(x, heads, gamma, eps, cos, sin, pos, pairing)
    if mag is None:
        z = BC.norm_rope(x, heads, gamma, eps, None, None, None, pairing).reshape(x.shape[0], heads, -1)
        # |a cos| + |b sin| <= |a| + |b|
        half = cos.shape[1]
        a = np.arange(half) if pairing == "halves" else np.arange(0, 2 * half, 2)
        b = a + (half if pairing == "halves" else 1)
        m = np.abs(z).copy()
        m[..., a] = m[..., b] = np.abs(z[..., a]) + np.abs(z[..., b])
        mag = m.reshape(x.shape[0], -1)
    return y, torch.finfo(FP[fp]).eps / 2 * np.abs(y) + 16 * 2.0 ** -24 * np.abs(mag) + 2.0 ** -25 * (fp == "f16")


@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("rows,nq,nkv,dh,rot,norm", [
    (1, 1, 1, 64, 64, True), (3, 5, 2, 128, 128, True), (67, 32, 8, 128, 64, True), (5, 7, 7, 64, 16, False), (9, 4, 1, 256, 256, True),
    (4, 3, 1, 80, 32, True), (2, 3, 2, 96, 96, True), (6, 2, 1, 16, 16, True), (3, 6, 3, 32, 16, True), (5, 9, 3, 208, 208, False), (4, 4, 2, 128, 0, True)])
def test_norm_and_rotation(h, fp, pairing, rows, nq, nkv, dh, rot, norm):
    g = np.random.default_rng(rows + dh)
    qt, qx = to_fp(g.standard_normal((rows, nq * dh)) * 3, fp)
    kt, kx = to_fp(g.standard_normal((rows, nkv * dh)) * 0.01, fp)
    gq, gk = (1 + 0.2 * g.standard_normal(dh)).astype(np.float32), (1 + 0.2 * g.standard_normal(dh)).astype(np.float32)
    c, s, ct, st = _tables(500, rot) if rot else (None,) * 4
    pos = g.integers(0, 500, rows).astype(np.int32)
    qo, ko = torch.full_like(qt, 9.0), torch.full_like(kt, 9.0)
    h.hero_qk_norm_rope(hero.tensor(qt), hero.tensor(kt), hero.tensor(qo), hero.tensor(ko), nq, nkv, torch.from_numpy(pos).cuda() if rot else None, ct, st,
                        torch.from_numpy(gq).cuda() if norm else None, torch.from_numpy(gk).cuda() if norm else None, 1e-5, pairing)
    h.check()
    for got, x, heads, gm in ((qo, qx, nq, gq), (ko, kx, nkv, gk)):
        y, bar = _bound(x, heads, gm if norm else None, 1e-5, c, s, pos, pairing, fp)
        assert np.all(np.abs(got.double().cpu().numpy() - y) <= bar)


def test_strided_in_place_norm_of_queries_only_and_far_positions(h):
    rows, nq, nkv, dh = 33, 6, 2, 128
    g = np.random.default_rng(5)
    w = (nq + 2 * nkv) * dh
    t, x = to_fp(g.standard_normal((rows, w)), "bf16")
    c, s, ct, st = _tables(131072, dh)
    pos = np.array([131071 - i for i in range(rows)], np.int32)
    gm = np.ones(dh, np.float32) * 0.5
    q, k = t[:, :nq * dh], t[:, nq * dh:(nq + nkv) * dh]
    h.hero_qk_norm_rope(hero.tensor(q), hero.tensor(k), hero.tensor(q), hero.tensor(k), nq, nkv, torch.from_numpy(pos).cuda(), ct, st,
                        torch.from_numpy(gm).cuda(), None)
    h.check()
    y, bar = _bound(x[:, :nq * dh], nq, gm, 1e-6, c, s, pos, "halves", "bf16")
    assert np.all(np.abs(q.double().cpu().numpy() - y) <= bar)
    y, bar = _bound(x[:, nq * dh:(nq + nkv) * dh], nkv, None, 1e-6, c, s, pos, "halves", "bf16")
    assert np.all(np.abs(k.double().cpu().numpy() - y) <= bar)
    assert np.array_equal(t[:, (nq + nkv) * dh:].double().cpu().numpy(), x[:, (nq + nkv) * dh:])         # the values are not touched


def test_queries_alone_and_int8_outputs_feed_the_attention_core(h):
    # q and k as the INT8 operands of hero_int8_attention: codes within one of the fp64 quotient's rounding only at ties
    rows, nq, dh = 20, 4, 64
    g = np.random.default_rng(6)
    qt, qx = to_fp(g.standard_normal((rows, nq * dh)), "f16")
    c, s, ct, st = _tables(64, dh)
    pos = np.arange(rows, dtype=np.int32)
    sc = torch.tensor([0.03], device="cuda")
    qo = torch.zeros(rows, nq * dh, dtype=torch.int8, device="cuda")
    h.hero_qk_norm_rope(hero.tensor(qt), None, hero.tensor(qo, "sq", sc), None, nq, 0, torch.from_numpy(pos).cuda(), ct, st,
                        torch.ones(dh, device="cuda"))
    h.check()
    y = BC.norm_rope(qx, nq, np.ones(dh), 1e-6, c, s, pos, "halves") / float(sc[0])
    got = qo.double().cpu().numpy()
    # half a step, plus FP32 noise of a value of at most 8 sigma / 0.03
    assert np.all(np.abs(got - np.clip(y, -127, 127)) <= 0.5 + 32 * 2.0 ** -24 * 300)


def test_a_row_of_zeros_and_one_without_a_norm_of_large_values(h):
    dh = 64
    x = np.zeros((2, dh))
    x[1] = 6e4
    t, xr = to_fp(x, "f16")
    out = torch.ones_like(t)
    h.hero_qk_norm_rope(hero.tensor(t), None, hero.tensor(out), None, 1, 0, q_gamma=torch.ones(dh, device="cuda"))
    h.check()
    y, bar = _bound(xr, 1, np.ones(dh), 1e-6, None, None, None, "halves", "f16")
    assert np.all(np.abs(out.double().cpu().numpy() - y) <= bar) and torch.all(out[0] == 0)


def test_positions_outside_the_tables_are_clamped_and_reported(h):
    dh = 64
    t, xr = to_fp(np.random.default_rng(1).standard_normal((3, dh)), "bf16")
    c, s, ct, st = _tables(10, dh)
    pos = np.array([-1, 4, 10], np.int32)
    out = torch.empty_like(t)
    h.hero_qk_norm_rope(hero.tensor(t), None, hero.tensor(out), None, 1, 0, torch.from_numpy(pos).cuda(), ct, st)
    with pytest.raises(hero.HeroError, match="position") as e:
        h.check()
    assert e.value.status == hero.ERR_INVALID_ARG
    y, bar = _bound(xr, 1, None, 0, c, s, pos, "halves", "bf16")
    assert np.all(np.abs(out.double().cpu().numpy() - y) <= bar)


def test_binding_refusals(h):
    t = hero.tensor(torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda"))
    c = torch.zeros(4, 32, device="cuda")
    pos = torch.zeros(3, dtype=torch.int32, device="cuda")
    for kw in (dict(cos=c, sin=c), dict(cos=c, sin=c[:, :16], pos=pos), dict(cos=c, sin=c, pos=pos[:2]), dict(cos=c, sin=c, pos=pos.long()),
               dict(q_gamma=c[0, :16]), dict(cos=c.cpu(), sin=c, pos=pos), dict(cos=c.double(), sin=c.double(), pos=pos)):
        with pytest.raises(hero.HeroError):
            h.hero_qk_norm_rope(t, None, t, None, 1, 0, **kw)
