"""GPU: hero_moe_linear against the oracle, over ragged groups, types, activations and strides; its observer, bounds on the device and refusals."""
import numpy as np
import pytest
import torch

from oracle import moe as M
from paper_2310_17723_b200 import hero
from moe_util import FP, Q8, STEP, assert_near, deal, f32, linear_bounds, num, to

pytestmark = pytest.mark.gpu

SPREAD = {"i8": 36.0, "f8": 60.0, "bf16": 1.0, "f16": 1.0}


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def filled(rows, cols, kind, pad):
    """An output of a recognisable value, with pad more columns in its rows."""
    wide = torch.full((rows, cols + pad), 3.0, device="cuda").to(Q8.get(kind) or FP[kind])
    return wide, wide[:, :cols]


def case(h, seed, kind, counts, N, K, act="none", gated=False, gather=True, out="bf16", bias=True, post=True, pad=0, tail=0, T=None, twq=True, observe=False):
    g = np.random.default_rng(seed)
    E, q8 = len(counts), kind in Q8
    T = T or max(1, sum(counts) // 3)
    offset, token, offset_t, token_t = deal(g, counts, T, tail)
    R = len(token)
    rows = T if gather else R
    at, a = to(g.standard_normal((rows, K)) * SPREAD[kind], kind)
    wt, w = to(g.standard_normal((E, N, K)) * SPREAD[kind] / (1 if q8 else np.sqrt(K)), kind)
    if pad:                                                 # wider strides everywhere
        wide = torch.zeros(rows, K + 32, dtype=at.dtype, device="cuda")
        wide[:, :K].view(torch.int8 if q8 else at.dtype).copy_(at.view(torch.int8) if q8 else at)
        at = wide[:, :K]
        deep = torch.zeros(E, N + 3, K + 16, dtype=wt.dtype, device="cuda")
        deep[:, :N, :K].view(torch.int8 if q8 else wt.dtype).copy_(wt.view(torch.int8) if q8 else wt)
        wt = deep[:, :N, :K]
    rs_t, rs = f32(np.exp(0.3 * g.standard_normal(rows)) / SPREAD[kind]) if q8 and twq else (None, None)
    cs_t, cs = f32(np.exp(0.3 * g.standard_normal((E, N))) / (SPREAD[kind] * np.sqrt(K)) * (1 if twq else 1 / SPREAD[kind])) if q8 else (None, None)
    b_t, b = f32(0.5 * g.standard_normal((E, N))) if bias else (None, None)
    n_out = N // 2 if gated else N
    size = {"i8": 40.0, "f8": 60.0}.get(out, 1.0)
    post_t, post_n = f32(size * np.exp(0.3 * g.standard_normal((E, n_out)))) if post else (None, None)
    wide, y_t = filled(max(R, 1), n_out, out, 32 if pad else 0)
    y_t = y_t[:R]
    seen = torch.zeros(E, n_out, device="cuda") if observe else None
    h.hero_moe_linear(hero.tensor(at, "twq", rs_t) if rs_t is not None else hero.tensor(at), wt, hero.tensor(y_t), offset_t, token=token_t if gather else None,
                      w_scale=cs_t, bias=b_t, act=act, gated=gated, post_scale=post_t, out_col_absmax=seen)
    h.check()
    y, v, size = M.linear(a, rs, w, cs, b, act, gated, post_n, offset, token if gather else None)
    bar = linear_bounds(y, v, size, act, gated, post_n, kind, K, offset)
    got = num(y_t)
    assert_near(got[:offset[-1]], y, bar, out, (kind, act, gated, out))
    assert np.all(got[offset[-1]:] == 3.0) and np.all(num(wide)[:, n_out:] == 3.0)       # nobody's rows and columns
    if observe:
        want = np.stack([np.abs(got[offset[e]:offset[e + 1]]).max(0, initial=0.0) for e in range(E)])
        assert np.array_equal(num(seen), want)
    return y_t


RAGGED = [0, 1, 15, 16, 17, 0, 31, 33, 64, 65, 3, 130, 0]            # 375 rows, 13 experts: few rows each
FULL = [255, 0, 256, 257, 1, 300, 513]                               # tiles of up to 256 rows, the rest dealt evenly
LONE = [0] * 30 + [300] + [0] * 15 + [70] + [0] * 20                 # few rows on average, many in two experts


@pytest.mark.parametrize("counts", [RAGGED, FULL, LONE], ids=["ragged", "full", "lone"])
@pytest.mark.parametrize("kind,out", [("i8", "i8"), ("i8", "bf16"), ("i8", "f16"), ("f8", "f8"), ("f8", "bf16"), ("bf16", "bf16"), ("f16", "i8"), ("f16", "f16"), ("bf16", "f8")])
@pytest.mark.parametrize("act,gated", [("none", False), ("silu", True), ("gelu_erf", False), ("gelu_tanh", True)])
def test_types_and_activations(h, counts, kind, out, act, gated):
    case(h, 11, kind, counts, 288, 208, act, gated, out=out, tail=5)


@pytest.mark.parametrize("counts", [RAGGED, FULL], ids=["ragged", "full"])
@pytest.mark.parametrize("N,K,gated", [(16, 16, False), (32, 16, True), (48, 128, False), (160, 144, True), (272, 1040, False), (544, 336, True), (528, 80, False), (1056, 640, True)])
@pytest.mark.parametrize("kind", ["i8", "bf16"])
def test_sizes(h, counts, N, K, gated, kind):
    if kind == "bf16":
        K = K // 2 if K > 16 else 8
    case(h, 12, kind, counts, N, K, "silu" if gated else "none", gated, out="i8" if kind == "i8" else "bf16", pad=1)


@pytest.mark.parametrize("counts", [RAGGED, FULL], ids=["ragged", "full"])
@pytest.mark.parametrize("kw", [dict(gather=False, tail=3), dict(bias=False), dict(post=False), dict(twq=False), dict(bias=False, post=False, act="silu"),
                                dict(gather=False, gated=True, act="none"), dict(act="silu"), dict(act="gelu_erf", gated=True), dict(T=1)])
def test_what_may_be_absent(h, counts, kw):
    case(h, 13, "i8", counts, 160, 256, **dict(dict(out="f16"), **kw))


@pytest.mark.parametrize("counts", [[1], [7], [0], [0, 0, 2], [1] * 40, [0] * 511 + [4], [2] * 512, [1000], [3, 2000]])
def test_groups(h, counts):
    case(h, 14, "i8", counts, 96, 96, out="i8", tail=2, T=9)
    case(h, 15, "i8", counts, 64, 96, "silu", True, out="bf16", tail=2, T=9)


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("counts", [RAGGED, FULL], ids=["ragged", "full"])
def test_observer(h, counts, gated):
    case(h, 16, "bf16", counts, 192, 128, "silu", gated, out="f16", observe=True, tail=4)
    case(h, 17, "i8", counts, 192, 128, "none", gated, out="bf16", observe=True)


@pytest.mark.parametrize("M_rows", [5, 40, 300])
@pytest.mark.parametrize("act", ["none", "gelu_erf"])
@pytest.mark.parametrize("out", [torch.int8, torch.float16])
def test_one_expert_is_the_dense_linear_bit_for_bit(h, M_rows, act, out):
    g = np.random.default_rng(18)
    N, K = 272, 400
    at, wt = to(g.standard_normal((M_rows, K)) * 36, "i8")[0], to(g.standard_normal((1, N, K)) * 36, "i8")[0]
    rs, cs, b, post = (f32(x)[0] for x in (g.uniform(0.5, 2, M_rows) / 36, g.uniform(0.5, 2, (1, N)) / 720, g.standard_normal((1, N)), g.uniform(20, 50, (1, N))))
    y = [torch.zeros(M_rows, N, dtype=out, device="cuda") for _ in range(2)]
    h.hero_moe_linear(hero.tensor(at, "twq", rs), wt, hero.tensor(y[0]), torch.tensor([0, M_rows], dtype=torch.int32, device="cuda"), w_scale=cs, bias=b, act=act, post_scale=post)
    h.hero_w8a8_linear(hero.tensor(at, "twq", rs), wt[0], hero.tensor(y[1]), w_scale=cs[0], bias=b[0], act=act, post_scale=post[0])
    h.check()
    assert torch.equal(y[0], y[1])


def test_rows_with_infinities_and_nan_stay_among_themselves(h):
    # a token that is infinite or NaN reaches its own rows alone
    g = np.random.default_rng(19)
    counts, K, N = [20, 0, 40, 300], 64, 96
    offset, token, offset_t, token_t = deal(g, counts, 50)
    at, a = to(g.standard_normal((50, K)), "bf16")
    wt, w = to(g.standard_normal((4, N, K)) / 8, "bf16")
    at[7, 3], at[9, 5] = float("nan"), float("inf")
    y = torch.zeros(360, N, dtype=torch.bfloat16, device="cuda")
    h.hero_moe_linear(hero.tensor(at), wt, hero.tensor(y), offset_t, token=token_t)
    h.check()
    a[[7, 9]] = 0
    want, v, size = M.linear(a, None, w, None, None, "none", False, None, offset, token)
    got, odd = num(y), np.isin(token, [7, 9])
    assert np.all(np.isnan(got[token == 7])) and not np.any(np.isfinite(got[token == 9]))
    bar = linear_bounds(want, v, size, "none", False, None, "bf16", K, offset)
    assert_near(got[~odd], want[~odd], bar[~odd], "bf16")


@pytest.mark.parametrize("E", [3, 40])
def test_bounds_that_the_host_cannot_see(h, E):
    # (every out-of-range index is clamped or left out on the device before it is used)
    T, K, N, R = 10, 64, 64, 120
    at, wt = torch.ones(T, K, dtype=torch.int8, device="cuda"), torch.ones(E, N, K, dtype=torch.int8, device="cuda")
    cs = torch.ones(E, N, device="cuda")
    for offset, token, full in (([0, 50, 20] + [120] * (E - 2), 0, None), ([0, -5] + [10] * (E - 1), 0, None), ([0] * E + [R + 7], 0, None), ([0] + [R] * E, T, R), ([0] + [R] * E, -3, R)):
        y = torch.full((R, N), 3, dtype=torch.float16, device="cuda")
        h.hero_moe_linear(hero.tensor(at), wt, hero.tensor(y), torch.tensor(offset, dtype=torch.int32, device="cuda"),
                          token=torch.full((R,), token, dtype=torch.int32, device="cuda"), w_scale=cs)
        with pytest.raises(hero.HeroError) as e:
            h.check()
        assert e.value.status == hero.ERR_INVALID_ARG and "expert" in str(e.value)
        assert set(y.unique().tolist()) <= {3.0, 64.0}
        if full:
            assert torch.all(y == 64.0)
    h.check()


def test_refusals_of_the_binding(h):
    A, out = torch.zeros(4, 64, dtype=torch.int8, device="cuda"), torch.zeros(8, 96, dtype=torch.int8, device="cuda")
    W, s = torch.zeros(3, 96, 64, dtype=torch.int8, device="cuda"), torch.ones(3, 96, device="cuda")
    offset, token = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda")
    good = dict(W=W, offset=offset, token=token, w_scale=s)
    for bad in (dict(W=W[0]), dict(W=W[:, :, :32]), dict(W=W.cpu()), dict(W=W.to(torch.bfloat16)), dict(W=W.transpose(1, 2)), dict(offset=offset[:3]),
                dict(offset=offset.long()), dict(token=token[:7]), dict(w_scale=s[:2]), dict(w_scale=s.half()), dict(bias=s[:, :90]), dict(post_scale=s[:, :48]),
                dict(w_scale=None), dict(act="silu", gated=True)):
        with pytest.raises(hero.HeroError):
            h.hero_moe_linear(hero.tensor(A), out=hero.tensor(out), **dict(good, **bad))
    h.check()


@pytest.mark.parametrize("gated", [False, True])
def test_long_runs_of_ragged_tiles_repeat_themselves(h, gated):
    # many tiles per CTA with few rows between full ones, in both forms of the kernel, launched behind one another and as a graph
    g = np.random.default_rng(20)
    K, N, E = 1040, 512, 64
    for top in (600, 40):
        counts = g.integers(0, top, E) * (g.random(E) < 0.8)
        counts[:3] = 1, 257, 5
        offset, token, offset_t, token_t = deal(g, counts, 500)
        at, wt = to(g.standard_normal((500, K)) * 36, "i8")[0], to(g.standard_normal((E, N, K)) * 36, "i8")[0]
        cs = torch.full((E, N), 1 / (36 * 36 * np.sqrt(K)), device="cuda")
        ys = [torch.zeros(len(token), N // 2 if gated else N, dtype=torch.float16, device="cuda") for _ in range(2)]
        call = lambda y: h.hero_moe_linear(hero.tensor(at), wt, hero.tensor(y), offset_t, token=token_t, w_scale=cs, act="silu", gated=gated)  # noqa: E731
        call(ys[0])
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                for _ in range(20):
                    call(ys[1])
        for _ in range(20):
            graph.replay()
        h.check()
        assert torch.equal(*ys)
