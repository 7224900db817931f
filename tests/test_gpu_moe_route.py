"""GPU: hero_moe_route against the oracle: the choice and the order exactly, the weights within FP32's roundings."""
import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import hero
from moe_util import FP, f32, num

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


class Out:
    def __init__(self, h, T, E, k):
        i32 = dict(dtype=torch.int32, device="cuda")
        self.expert, self.row, self.token = torch.full((T, k), 77, **i32), torch.full((T, k), 77, **i32), torch.full((T * k,), -9, **i32)
        self.weight, self.offset = torch.full((T, k), 7.0, device="cuda"), torch.full((E + 1,), 77, **i32)
        self.workspace = torch.full((h.hero_moe_route_workspace_bytes(T, E, k),), 0xff, dtype=torch.uint8, device="cuda")

    def args(self):
        return self.expert, self.weight, self.offset, self.token, self.row


def check(o, x, k, **kw):
    e, w, offset, token, row = M.route(x, k, **kw)
    assert np.array_equal(o.expert.cpu().numpy(), e)
    assert np.array_equal(o.offset.cpu().numpy(), offset)
    got = o.token.cpu().numpy()
    assert np.array_equal(got[:offset[-1]], token) and np.all(got[offset[-1]:] == -9)      # rows in nobody's use stay as they were
    assert np.array_equal(o.row.cpu().numpy(), row)
    # expf 2 units, a difference of logits rounded (2^-24 of it, into the exponent), a sum of E terms in a tree of E / 32 + 5 levels, the quotients
    # and the scale half a unit each
    fin = np.where(np.isfinite(x), x, 0.0)
    spread = np.ptp(fin, axis=1)[:, None] + np.abs(fin).max(1)[:, None]
    bar = w * 2.0 ** -23 * (16 + x.shape[1] / 32 + spread) + 2.0 ** -140
    assert np.all(np.abs(num(o.weight) - w) <= bar)


def logits(g, T, E, dt):
    t = torch.from_numpy((g.standard_normal((T, E)) * 1.5).astype(np.float32)).to(FP[dt]).cuda()
    return t, num(t)


@pytest.mark.parametrize("T", [1, 2, 31, 33, 96, 97, 700])
@pytest.mark.parametrize("E,k", [(1, 1), (3, 3), (8, 2), (33, 5), (64, 8), (128, 16), (200, 6), (512, 8)])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
def test_sizes(h, T, E, k, dt):
    g = np.random.default_rng(T * 1000 + E)
    for score, renorm, biased in (("softmax", True, False), ("sigmoid", True, True), ("softmax", False, True), ("sigmoid", False, False), ("softmax", False, False)):
        xt, x = logits(g, T, E, dt)
        bt, b = f32(0.3 * g.standard_normal(E)) if biased else (None, None)
        o = Out(h, T, E, k)
        h.hero_moe_route(hero.tensor(xt), *o.args(), score=score, renorm=renorm, scale=1.5, select_bias=bt, workspace=o.workspace)
        h.check()
        check(o, x, k, score=score, renorm=renorm, scale=1.5, bias=b)


@pytest.mark.parametrize("T", [40, 300])
@pytest.mark.parametrize("dt", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_ties_masks_infinities_and_nan(h, T, dt, biased, score):
    g = np.random.default_rng(5)
    E, k = 70, 6
    x = g.integers(-3, 4, (T, E)) * 0.5                               # many equal logits, zeros of both signs among them
    x[::7] *= -1.0
    x[1] = 0.25                                                       # all equal
    x[2] = -np.inf
    x[3] = np.nan
    x[4, 5:] = -np.inf                                                # fewer left than are to be chosen
    x[5, ::2] = np.nan
    x[6, [3, 9, 69]] = np.inf
    x[7] = -60 + x[7]
    x[8] = np.array([-1e4, 1e4])[g.integers(0, 2, E)]
    xt = torch.from_numpy(x.astype(np.float32)).to(FP[dt]).cuda()
    x = num(xt)
    b = np.zeros(E)
    b[[0, 20]] = -np.inf, np.nan
    bt, b = f32(b) if biased else (None, None)
    for renorm in (True, False):
        o = Out(h, T, E, k)
        h.hero_moe_route(hero.tensor(xt), *o.args(), score=score, renorm=renorm, select_bias=bt, workspace=o.workspace)
        h.check()
        check(o, x, k, score=score, renorm=renorm, bias=b)


@pytest.mark.parametrize("T", [60, 130])
@pytest.mark.parametrize("biased", [False, True])
@pytest.mark.parametrize("few", [False, True])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_keys_that_fp32_cannot_tell_apart(h, score, few, biased, T):
    # logits a unit of FP32 apart where a unit of the score is far coarser, in falling order of the expert: rounded keys would tie.  All experts, or
    # (few) nine of them around the border of the choice
    E, k = 96, 7
    g = np.random.default_rng(6)
    base = g.uniform(2.0, 6.0, (T, 1)).astype(np.float32)
    x = base + np.arange(E, dtype=np.float32)[None] * np.spacing(base)
    if few:
        y = (base - 4 + g.standard_normal((T, E)) * 0.5).astype(np.float32)
        near = np.array([3, 90, 17, 64, 40, 33, 95, 8, 50])
        y[:, near] = x[:, near]
        y[:, [1, 2]] = base + 1                            # two that are clearly first
        x = y
    xt, x = f32(x)
    bt, b = f32(np.full(E, 0.125)) if biased else (None, None)
    o = Out(h, T, E, k)
    h.hero_moe_route(hero.tensor(xt), *o.args(), score=score, select_bias=bt, workspace=o.workspace)
    h.check()
    check(o, x.astype(np.float64), k, score=score, bias=b)
    assert o.expert[0].tolist() == ([1, 2, 95, 90, 64, 50, 40] if few else [95, 94, 93, 92, 91, 90, 89])


@pytest.mark.parametrize("T", [50, 1000])
@pytest.mark.parametrize("n", [-3, 0, 1, 33, 50, 9999])
def test_padded_batch_and_strides(h, T, n):
    g = np.random.default_rng(7)
    wide = torch.from_numpy(g.standard_normal((T, 41)).astype(np.float32)).cuda()
    xt = wide[:, 3:40]                                                # any pitch, aligned to an element alone
    o = Out(h, T, 37, 4)
    h.hero_moe_route(hero.tensor(xt), *o.args(), n_tokens=torch.tensor([n], dtype=torch.int32, device="cuda"), workspace=o.workspace)
    h.check()
    check(o, num(xt), 4, n_tokens=n)


def test_no_tokens(h):
    o = Out(h, 0, 9, 2)
    h.hero_moe_route(hero.tensor(torch.zeros(0, 9, device="cuda")), *o.args())
    h.check()
    assert o.offset.tolist() == [0] * 10


def test_one_expert_takes_everything(h):
    T, E = 3000, 5
    x = torch.zeros(T, E, device="cuda")
    x[:, 3] = 1.0
    o = Out(h, T, E, 1)
    h.hero_moe_route(hero.tensor(x), *o.args(), workspace=o.workspace)
    h.check()
    assert o.offset.tolist() == [0, 0, 0, 0, T, T] and torch.equal(o.token.cpu(), torch.arange(T, dtype=torch.int32))


def test_refusals_of_the_binding(h):
    T, E, k = 8, 16, 2
    x = torch.zeros(T, E, device="cuda")
    o = Out(h, T, E, k)
    good = dict(expert=o.expert, weight=o.weight, offset=o.offset, token=o.token, row=o.row)
    for bad in (dict(expert=o.expert[:4]), dict(weight=o.weight.double()), dict(offset=o.offset[:E]), dict(token=o.token[:T]), dict(row=o.row.cpu()),
                dict(row=o.row.t().contiguous().t()), dict(select_bias=torch.zeros(E - 1, device="cuda")), dict(n_tokens=torch.zeros(2, dtype=torch.int32, device="cuda")),
                dict(n_tokens=torch.zeros(1, device="cuda"))):
        with pytest.raises(hero.HeroError):
            h.hero_moe_route(hero.tensor(x), **dict(good, **bad))
    h.check()
