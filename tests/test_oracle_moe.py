"""The oracle of the mixture of experts against library float64 routines, and the entry points' refusals, which need no GPU because they come before
anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import build as B
from paper_2310_17723_b200 import hero


def test_route_against_library_topk():
    g = np.random.default_rng(1)
    x = g.standard_normal((37, 19))
    for score in ("softmax", "sigmoid"):
        s = torch.softmax(torch.from_numpy(x), -1) if score == "softmax" else torch.sigmoid(torch.from_numpy(x))
        for bias in (None, g.standard_normal(19)):
            key = torch.from_numpy(x) if bias is None else s + torch.from_numpy(bias)
            ids = torch.topk(key, 5, -1)[1].numpy()
            for renorm in (False, True):
                e, w, offset, token, row = M.route(x, 5, score, renorm, 2.0, bias)
                assert np.array_equal(e, ids)
                want = np.take_along_axis(s.numpy(), ids, 1)
                want = 2.0 * (want / want.sum(1, keepdims=True) if renorm else want)
                assert np.allclose(w, want, rtol=1e-12)
                assert offset[-1] == 37 * 5 and np.array_equal(np.diff(offset), np.bincount(e.reshape(-1), minlength=19))
                for t in range(37):
                    for j in range(5):
                        assert token[row[t, j]] == t and offset[e[t, j]] <= row[t, j] < offset[e[t, j] + 1]
                for i in range(19):
                    assert np.all(np.diff(token[offset[i]:offset[i + 1]]) > 0)


def test_route_edges():
    inf, nan = np.inf, np.nan
    x = np.array([[1.0, 1.0, 1.0, 1.0], [-inf, 2.0, nan, -inf], [-inf, -inf, nan, -inf], [inf, 0.0, inf, 1.0], [-800.0, -801.0, -inf, -inf]])
    e, w, offset, token, row = M.route(x, 2, "softmax", False)
    assert e.tolist() == [[0, 1], [1, -1], [-1, -1], [0, 2], [0, 1]]
    assert np.allclose(w[:4], [[.25, .25], [1, 0], [0, 0], [.5, .5]]) and row[2].tolist() == [-1, -1]
    assert offset.tolist() == [0, 3, 6, 7, 7] and token.tolist() == [0, 3, 4, 0, 1, 4, 3]
    assert np.allclose(M.route(x, 2, "sigmoid", True)[1][4], [1 / (1 + np.exp(-1)), 1 / (1 + np.exp(1))])       # ratios survive
    assert M.route(x, 2, n_tokens=1)[0].tolist() == [[0, 1]] + [[-1, -1]] * 4
    assert M.route(x[:1], 2, bias=[0, -inf, 0.5, nan])[0].tolist() == [[2, 0]]


def test_linear_against_the_library_routine():
    g = np.random.default_rng(2)
    offset, token = np.array([0, 3, 3, 7]), np.array([4, 0, 2, 1, 1, 3, 0])
    a, W, b, cs, rs, post = (g.standard_normal(s) for s in ((5, 8), (3, 12, 8), (3, 12), (3, 12), (5,), (3, 6)))
    F = torch.nn.functional
    for act, f in (("gelu_erf", F.gelu), ("gelu_tanh", lambda v: F.gelu(v, approximate="tanh")), ("silu", F.silu)):
        y, _, _ = M.linear(a, rs, W, cs, b, act, True, post, offset, token)
        for e in range(3):
            for r in range(offset[e], offset[e + 1]):
                v = F.linear(torch.from_numpy(a[token[r]] * rs[token[r]]), torch.from_numpy(W[e] * cs[e][:, None]), torch.from_numpy(b[e]))
                assert np.allclose(y[r], (f(v[:6]) * v[6:]).numpy() * post[e], rtol=1e-10, atol=1e-12)


# ------------------------------------------------------------------------------------------------ refusals
@pytest.fixture(scope="module")
def call():
    """Calls an entry point with a blank handle: every refusal is made before the handle's device is looked at."""
    B.build()
    blank = (C.c_uint8 * (1 << 20))()

    def run(name, *structs):
        return getattr(hero.lib(), name)(C.cast(blank, C.c_void_p), *[C.byref(s) for s in structs], None)
    return run


P = 1 << 20                      # a 16-byte aligned address that nothing looks at
REFUSED = (hero.ERR_INVALID_ARG, hero.ERR_UNSUPPORTED, hero.ERR_ALIGNMENT, hero.ERR_WORKSPACE)


def _t(rows, cols, dtype=hero.BF16, gran=0, scale=None, data=P, ld=None):
    return hero.Tensor(data, dtype, gran, rows, cols, cols if ld is None else ld, scale)


def _route(**kw):
    d = dict(logits=_t(8, 64, hero.F32), n_tokens=None, select_bias=None, top_k=4, score=0, renorm=1, scale=1.0, expert=P, weight=P, offset=P,
             token=P, row=P, workspace=None, workspace_bytes=0)
    d.update(kw)
    return hero.MoeRouteArgs(**d)


@pytest.mark.parametrize("kw", [dict(logits=_t(8, 64, hero.I8)), dict(logits=_t(8, 513)), dict(logits=_t(8, 0)), dict(logits=_t(8, 64, ld=63)),
                                dict(logits=_t(8, 64, data=None)), dict(logits=_t(8, 64, hero.F32, data=P + 2)), dict(logits=_t(8, 64, data=P + 1)),
                                dict(top_k=0), dict(top_k=17), dict(top_k=65), dict(logits=_t(8, 3), top_k=4), dict(score=2), dict(expert=None),
                                dict(weight=None), dict(offset=None), dict(token=None), dict(row=None), dict(logits=_t(1 << 30, 64), top_k=2),
                                dict(logits=_t(-1, 64))])
def test_bad_routes_are_refused(call, kw):
    assert call("hero_moe_route", _route(**kw)) in REFUSED


def _linear(**kw):
    d = dict(A=_t(8, 64, hero.I8, 1, P), token=P, offset=P, W=P, N=96, ldw=64, expert_stride=96 * 64, n_experts=4, w_scale=P, bias=P, act=0,
             gated=0, post_scale=P, out=_t(16, 96, hero.I8), out_col_absmax=None)
    d.update(kw)
    return hero.MoeLinearArgs(**d)


@pytest.mark.parametrize("kw", [dict(A=_t(8, 64, hero.F32)), dict(A=_t(8, 72, hero.I8, 1, P, ld=80)), dict(A=_t(8, 64, hero.I8, 1, None)),
                                dict(A=_t(8, 64, hero.I8, 1, P, data=P + 8)), dict(A=_t(8, 64, hero.I8, 1, P, ld=72)), dict(N=100), dict(N=0),
                                dict(gated=1, N=80, out=_t(16, 40)), dict(gated=1), dict(gated=2), dict(W=None), dict(W=P + 4), dict(ldw=63), dict(ldw=72),
                                dict(expert_stride=8), dict(expert_stride=6152), dict(n_experts=0), dict(n_experts=513), dict(w_scale=None),
                                dict(act=4), dict(act=-1), dict(out=_t(16, 80, hero.I8)), dict(out=_t(16, 96, hero.F8)), dict(out=_t(16, 96, hero.F32)),
                                dict(out=_t(16, 96, hero.I32)), dict(out=_t(16, 96, hero.I8, 1, P)), dict(out=_t(16, 96, hero.I8, data=P + 2)),
                                dict(A=_t(8, 64, hero.F8, 1, P)), dict(token=None), dict(offset=None), dict(out_col_absmax=P),
                                dict(A=_t(0, 64, hero.I8, 1, P)), dict(ldw=1 << 37), dict(expert_stride=1 << 38)])
def test_bad_products_are_refused(call, kw):
    assert call("hero_moe_linear", _linear(**kw)) in REFUSED


def _combine(**kw):
    d = dict(y=_t(16, 64), row=P, weight=P, expert=None, top_k=2, n_experts=0, residual=_t(8, 64), shared=_t(0, 0, 0, data=None), gamma=P, beta=P, eps=1e-5,
             out=_t(8, 64, hero.I8, 1, P), fp_out=_t(8, 64))
    d.update(kw)
    return hero.MoeCombineArgs(**d)


NONE = _t(0, 0, 0, data=None)


@pytest.mark.parametrize("kw", [dict(y=_t(16, 80)), dict(y=_t(16, 64, hero.F32)), dict(y=NONE), dict(y=_t(16, 64, hero.I8, 1, P)), dict(row=None),
                                dict(weight=None), dict(y=_t(16, 64, hero.I8, 2, P)), dict(y=_t(16, 64, hero.I8, 2, P), expert=P),
                                dict(y=_t(16, 64, hero.I8, 2, P + 4), expert=P, n_experts=4), dict(top_k=0), dict(top_k=17), dict(residual=_t(7, 64)),
                                dict(residual=_t(8, 64, hero.F32)), dict(residual=_t(8, 64, data=P + 2)), dict(shared=_t(8, 80)), dict(gamma=None),
                                dict(beta=None), dict(gamma=P + 4), dict(out=_t(8, 64, hero.I8)), dict(out=_t(8, 64, hero.F32)),
                                dict(out=NONE, fp_out=NONE), dict(fp_out=_t(8, 64, hero.I8, 1, P)), dict(fp_out=_t(9, 64)),
                                dict(out=_t(8, 72), fp_out=NONE, residual=NONE, y=_t(16, 72)), dict(out=_t(8, 16400), fp_out=NONE, residual=NONE, y=_t(16, 16400))])
def test_bad_sums_are_refused(call, kw):
    assert call("hero_moe_combine", _combine(**kw)) in REFUSED


def test_a_workspace_that_is_missing_or_too_small_is_refused():
    B.build()
    # a handle of a device with 148 SMs: device, sm_count are its first two fields
    blank = (C.c_uint8 * (1 << 20))()
    C.cast(blank, C.POINTER(C.c_int))[1] = 148
    h, n, need = C.cast(blank, C.c_void_p), C.c_size_t(), []
    for T in range(0, 400000, 997):
        assert hero.lib().hero_moe_route_workspace_bytes(h, T, 64, 4, C.byref(n)) == hero.OK
        need.append(n.value)
        if n.value:
            for ws, size in ((None, 0), (P, n.value - 1), (P + 4, n.value)):
                a = _route(logits=_t(T, 64), workspace=ws, workspace_bytes=size)
                assert hero.lib().hero_moe_route(h, C.byref(a), None) in (hero.ERR_WORKSPACE, hero.ERR_ALIGNMENT)
    assert need == sorted(need) and need[0] == 0 and need[-1] > 0
    for T, E, k in ((-1, 64, 4), (8, 0, 1), (8, 513, 1), (8, 64, 17), (8, 4, 5), (1 << 31, 64, 1)):
        assert hero.lib().hero_moe_route_workspace_bytes(h, T, E, k, C.byref(n)) == hero.ERR_UNSUPPORTED


def test_nothing_to_do_is_no_error(call):
    assert call("hero_moe_linear", _linear(out=_t(0, 96, hero.I8, data=None))) == hero.OK
    empty = dict(residual=_t(0, 64, data=None), out=_t(0, 64, hero.I8, 1, P, data=None), fp_out=_t(0, 64, data=None))
    assert call("hero_moe_combine", _combine(**empty)) == hero.OK


def test_struct_sizes_match_the_compiler():
    assert C.sizeof(hero.MoeRouteArgs) == 48 + 2 * 8 + 4 * 4 + 5 * 8 + 2 * 8
    assert C.sizeof(hero.MoeLinearArgs) == 48 + 3 * 8 + 3 * 8 + 8 + 2 * 8 + 8 + 8 + 48 + 8      # n_experts is followed by 4 bytes of padding
    assert C.sizeof(hero.MoeCombineArgs) == 48 + 3 * 8 + 8 + 2 * 48 + 2 * 8 + 8 + 2 * 48        # eps too


def test_silu_belongs_to_the_experts_alone(call):
    a = hero.LinearArgs(_t(8, 64, hero.I8), P, 96, 64, P, None, hero.ACT_SILU, None, _t(8, 96, hero.I8), None)
    assert call("hero_w8a8_linear", a) == hero.ERR_INVALID_ARG
