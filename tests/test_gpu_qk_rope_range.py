"""GPU parity of hero_qk_norm_rope where values are not finite or leave the range of the INT8 output, and of its INT8 outputs for
keys, both pairings and a scale for each output.  Bounds as in test_gpu_qk_rope.py."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero
from block_util import to_fp
from test_gpu_qk_rope import _tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("dh,rot", [(128, 64), (64, 0), (80, 32), (256, 128)])
@pytest.mark.parametrize("norm", [False, True])
def test_what_is_not_finite_stays_where_the_definition_leaves_it(h, fp, pairing, dh, rot, norm):
    # infinities and NaN in features that pass through and in features that turn, zeros of either sign; a row each, and one of all
    g = np.random.default_rng(dh + rot)
    rows, nq = 6, 3
    x = g.standard_normal((rows, nq, dh))
    x[:, :, 5 % max(rot, 8)] = -0.0
    x[:, :, dh - 3] = -0.0
    x[0, 0, dh - 6] = np.inf
    x[1, 1, dh - 7] = np.nan
    x[2, 2, [dh - 1, dh - 2]] = -np.inf, np.inf
    x[3, 0, 2] = np.inf                                        # turned where there is a rotation
    x[4, 1, 1] = np.nan
    x[5, :, dh - 5], x[5, 0, 0] = np.inf, -np.inf
    t, xr = to_fp(x.reshape(rows, nq * dh), fp)
    c, s, ct, st = _tables(50, rot, seed=0.3) if rot else (None,) * 4
    pos = g.integers(0, 50, rows).astype(np.int32)
    gm = (1 + 0.2 * g.standard_normal(dh)).astype(np.float32) if norm else None
    out = torch.zeros_like(t)
    h.hero_qk_norm_rope(hero.tensor(t), None, hero.tensor(out), None, nq, 0, torch.from_numpy(pos).cuda() if rot else None, ct, st,
                        torch.from_numpy(gm).cuda() if norm else None, pairing=pairing)
    h.check()
    with np.errstate(invalid="ignore"):
        want = BC.norm_rope(xr, nq, gm, 1e-6, c, s, pos, pairing)
        size = np.abs(BC.norm_rope(np.where(np.isfinite(xr), xr, 0.0), nq, gm, 1e-6, None, None, None, pairing)).max()
    got = out.double().cpu().numpy()
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[np.isinf(want)], want[np.isinf(want)]) and np.array_equal(np.isinf(got), np.isinf(want))
    fin = np.isfinite(want)
    # half a step of the type, and 16 units of 2^-24 on the two products, each at most the largest magnitude
    assert np.all(np.abs(got - want)[fin] <= torch.finfo(t.dtype).eps / 2 * np.abs(want[fin]) + 32 * 2.0 ** -24 * size + 2.0 ** -25)
    if not norm:                                               # what passes through is the input, signs of zeros and all
        a, b = (y.view(torch.int16).reshape(rows, nq, dh)[..., rot:] for y in (out, t))
        keep = ~torch.isnan(t.reshape(rows, nq, dh)[..., rot:])
        assert torch.equal(a[keep], b[keep])


@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
def test_int8_outputs_saturate(h, pairing):
    # infinities, and quotients beyond FP32: the largest code of their sign
    rows, dh, rot = 4, 64, 32
    g = np.random.default_rng(1)
    x = g.standard_normal((rows, 2 * dh))
    x[0, [40, 41, 63]] = np.inf, -np.inf, np.inf               # pass through
    x[1, [dh + 33, dh + 50]] = 3e38, -3e38
    x[2] *= 1e30
    x[3, 10] = np.inf                                          # turned: its pair is infinite
    t, xr = to_fp(x, "bf16")
    c, s, ct, st = _tables(50, rot, seed=0.3)
    pos = np.array([3, 7, 11, 19], np.int32)
    for step in (0.02, 1e-5, 1e-25, 1e-35):
        out = torch.zeros(rows, 2 * dh, dtype=torch.int8, device="cuda")
        sc = torch.tensor([step], device="cuda")
        h.hero_qk_norm_rope(hero.tensor(t), None, hero.tensor(out, "sq", sc), None, 2, 0, torch.from_numpy(pos).cuda(), ct, st, pairing=pairing)
        h.check()
        y = BC.norm_rope(xr, 2, None, 0.0, c, s, pos, pairing)
        sign = BC.to_codes(np.clip(y / float(sc[0]), -1e9, 1e9), "i8")
        far = np.abs(y) > 200 * step
        assert np.array_equal(out.double().cpu().numpy()[far], sign[far]), step


@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("dh,rot,nq,nkv", [(128, 128, 8, 2), (64, 32, 3, 3), (96, 96, 2, 1)])
def test_int8_queries_and_keys_with_a_scale_each(h, fp, pairing, dh, rot, nq, nkv):
    rows = 23
    g = np.random.default_rng(dh)
    (qt, qx), (kt, kx) = (to_fp(g.standard_normal((rows, n * dh)) * z, fp) for n, z in ((nq, 2.0), (nkv, 0.3)))
    c, s, ct, st = _tables(64, rot)
    pos = g.integers(0, 64, rows).astype(np.int32)
    gq, gk = ((1 + 0.2 * g.standard_normal(dh)).astype(np.float32) for _ in range(2))
    sq, sk = torch.tensor([0.021], device="cuda"), torch.tensor([0.034], device="cuda")
    qo, ko = (torch.zeros(rows, n * dh, dtype=torch.int8, device="cuda") for n in (nq, nkv))
    h.hero_qk_norm_rope(hero.tensor(qt), hero.tensor(kt), hero.tensor(qo, "sq", sq), hero.tensor(ko, "sq", sk), nq, nkv, torch.from_numpy(pos).cuda(),
                        ct, st, torch.from_numpy(gq).cuda(), torch.from_numpy(gk).cuda(), pairing=pairing)
    h.check()
    for got, x, heads, gm, sc in ((qo, qx, nq, gq, sq), (ko, kx, nkv, gk, sk)):
        y = BC.norm_rope(x, heads, gm, 1e-6, c, s, pos, pairing) / float(sc[0])
        # half a step; FP32 noise of 32 units of 2^-24 on two products of at most sqrt(dh) * 2 each over the scale
        assert np.all(np.abs(got.double().cpu().numpy() - np.clip(y, -127, 127)) <= 0.5 + 32 * 2.0 ** -24 * 4 * dh ** 0.5 / float(sc[0]))
    # one of the two in the input's type
    k16 = torch.zeros_like(kt)
    h.hero_qk_norm_rope(hero.tensor(qt), hero.tensor(kt), hero.tensor(qo, "sq", sq), hero.tensor(k16), nq, nkv, torch.from_numpy(pos).cuda(),
                        ct, st, torch.from_numpy(gq).cuda(), torch.from_numpy(gk).cuda(), pairing=pairing)
    h.check()
    y = BC.norm_rope(kx, nkv, gk, 1e-6, c, s, pos, pairing)
    got = k16.double().cpu().numpy()
    assert np.all(np.abs(got - y) <= torch.finfo(kt.dtype).eps / 2 * np.abs(y) + 32 * 2.0 ** -24 * 4 * dh ** 0.5 + 2.0 ** -25)


@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
@pytest.mark.parametrize("rot", [0, 32, 64])
def test_a_head_whose_squares_are_beyond_fp32_is_zeros(h, pairing, rot):
    # the definition is in FP32 throughout: an infinite mean of squares divides every finite feature to 0, whatever the gammas are
    dh, nq = 64, 3
    g = np.random.default_rng(2)
    x = g.standard_normal((2, nq, dh))
    x[0, 1], x[1, 2] = 3e38 * np.sign(x[0, 1]), 1e20 * x[1, 2]
    t, xr = to_fp(x.reshape(2, nq * dh), "bf16")
    c, s, ct, st = _tables(50, rot, seed=0.3) if rot else (None,) * 4
    pos = np.array([7, 31], np.int32)
    gm = g.uniform(1.5, 3.0, dh).astype(np.float32)
    out = torch.ones_like(t)
    h.hero_qk_norm_rope(hero.tensor(t), None, hero.tensor(out), None, nq, 0, torch.from_numpy(pos).cuda() if rot else None, ct, st,
                        torch.from_numpy(gm).cuda(), pairing=pairing)
    h.check()
    got = out.double().cpu().numpy().reshape(2, nq, dh)
    assert np.all(got[0, 1] == 0) and np.all(got[1, 2] == 0)
    want = BC.norm_rope(xr, nq, gm, 1e-6, c, s, pos, pairing).reshape(2, nq, dh)
    for at in ((0, 0), (0, 2), (1, 0), (1, 1)):
        assert np.all(np.abs(got[at] - want[at]) <= 2.0 ** -8 * np.abs(want[at]) + 32 * 2.0 ** -24 * np.abs(want[at]).max() * 2)
