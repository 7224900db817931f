"""GPU parity of hero_block_attention at the ends of its number range: value scales below FP32's normal numbers, values near the largest
and the smallest that BF16 holds, scores far below zero or so large that their own rounding counts, subnormal queries.  Each on the
kernel for few rows (one CTA per group, and shares that are joined) and on the one for many (whole, and keys in parts).  Bounds as in
test_gpu_block_attention.py; where an output is itself subnormal, half a step of it (2^-134 in BF16) is added."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero
from block_util import Cache, start_tensor, starts, to_fp
from test_gpu_block_attention import _compare, _expect, _q, _run

pytestmark = pytest.mark.gpu

LENS = [200, 150]
# (rows of each sequence, host-side bound on the lengths): few rows direct and in shares, many rows whole and in parts
FORMS = [([1, 1], 300), ([1, 1], 5000), ([6, 2], 5000), ([80, 60], 300), ([80, 60], 5000)]


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def _cache(kind, dh, max_len, k_scale=None, v_scale=None, page=16):
    c = Cache(7, kind, page, 1, dh, LENS, max_len=max_len)
    for x, s in (("k", k_scale), ("v", v_scale)):
        if s is not None:
            c.scale[x][:] = s
            _renew(c, x)
    return c


def _renew(c, x):
    c.scale_t[x].copy_(torch.from_numpy(c.scale[x]))


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
def test_value_scales_below_the_normal_range_beside_ordinary_ones(h, kind, dh, counts, max_len):
    # what the append makes of values of 1e-37: a scale whose reciprocal is beyond FP32; a page of zeros beside it, ordinary pages behind it
    c = _cache(kind, dh, max_len)
    for b in range(2):
        for i, pid in enumerate(c.table[b][:6]):
            c.scale["v"][pid] = 0.0 if i in (1, 4) else 1e-39 * (i + 1)
    _renew(c, "v")
    qt, qx = _q(1, sum(counts), 2 * dh, "bf16")
    _compare(c, _run(h, c, qt, counts, 2, "bf16"), qx, counts, 2, "bf16")


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("kind,dh", [("i8", 128), ("f8", 64)])
@pytest.mark.parametrize("unit", [5e35, 2.0 ** -130])
def test_values_near_the_ends_of_the_range(h, kind, dh, counts, max_len, unit):
    # sums of P V before their division by the row's sum are up to 2^15 keys times the values: FP32 does not hold them at one end, and
    # a factor divided by the row's sum loses its bits at the other
    g = np.random.default_rng(2)
    c = _cache(kind, dh, max_len)
    c.scale["v"][:] = unit * g.uniform(0.3, 1.0, c.scale["v"].shape)
    _renew(c, "v")
    qt, qx = _q(3, sum(counts), 2 * dh, "bf16")
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy()
    want, bar = _expect(c, qx, counts, 2, dh ** -0.5, sum(counts))
    # probabilities are held relative to the largest value scale, a normal number: 2^-36 of 2^-126 times the largest code per key; partial
    # results in FP32's subnormal numbers are off by 2^-150 each, sixteen of them at most
    bar = bar + max(LENS) * 2.0 ** -36 * 448 * 2.0 ** -126 + 16 * 2.0 ** -150
    bar = bar + torch.finfo(torch.bfloat16).eps / 2 * (np.abs(want) + bar) + 2.0 ** -134
    assert np.all(np.abs(got - want) <= bar), np.nanmax(np.abs(got - want) / bar)


def _one_loud_token(kind, dh, max_len, k_unit):
    """Keys of one sign in which token 3 of each sequence is small: against queries of the other sign its score is the largest by far."""
    c = _cache(kind, dh, max_len, k_scale=k_unit)
    codes = BC.to_codes(np.maximum(np.abs(c.codes["k"]), 50.0), kind)
    for b in range(2):
        codes[c.table[b][0], :, 3] = 1.0
    c.codes["k"] = codes
    c.buf["k"].copy_(torch.from_numpy(codes.astype(np.float32)).to(c.buf["k"].dtype))
    return c


def _is_the_value_of_its_one_token(h, kind, dh, counts, max_len, k_unit, q_unit):
    c = _one_loud_token(kind, dh, max_len, k_unit)
    rows = sum(counts)
    qt, _ = to_fp(-q_unit * np.random.default_rng(4).uniform(1.0, 1.5, (rows, 2 * dh)), "bf16")
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy()
    for b, (n, at) in enumerate(zip(counts, starts(counts))):
        want = np.tile(c.values("v", b)[3, 0], (n, 2))
        t = LENS[b] - n + np.arange(n)             # the rows' tokens: those before the loud one do not see it, rows without one are zeros
        assert np.all(got[at:at + n][t < 0] == 0)
        # half a step of BF16, and two roundings of FP16 (the probability and its product with the value scale)
        assert np.all((np.abs(got[at:at + n] - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want))[t >= 3]), b


@pytest.mark.parametrize("counts,max_len", FORMS[:3])
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
def test_few_rows_whose_scores_all_lie_below_a_large_negative_number(h, kind, dh, counts, max_len):
    # the largest score is about -1e32, the next fifty times as far
    _is_the_value_of_its_one_token(h, kind, dh, counts, max_len, 1e14, 1e17)


@pytest.mark.parametrize("counts,max_len", FORMS[:3])
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
@pytest.mark.parametrize("q_unit", [1e6, 3e6, 1e7, 2e7, 4e7, 1e9, 1e12])
def test_few_rows_whose_scores_are_rounded_by_more_than_the_probabilities_reach(h, kind, dh, counts, max_len, q_unit):
    # scores of 2^27: FP32 holds them in steps of 16, more than FP16 has above the place that the largest probability is given
    _is_the_value_of_its_one_token(h, kind, dh, counts, max_len, 1.0, q_unit)


@pytest.mark.parametrize("counts,max_len", FORMS[3:] + [([700, 60], 900)])
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
@pytest.mark.parametrize("k_unit,q_unit", [(1.0, 1e5), (1.0, 1e6), (1.0, 3e6), (1.0, 1e7), (1.0, 2e7), (1.0, 4e7), (1.0, 1e9), (1.0, 1e12), (1e14, 1e17)])
def test_many_rows_whose_scores_are_rounded_by_more_than_the_probabilities_reach(h, kind, dh, counts, max_len, k_unit, q_unit):
    _is_the_value_of_its_one_token(h, kind, dh, counts, max_len, k_unit, q_unit)


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("q_unit", [1.0, 1e3])
def test_keys_that_are_all_alike_share_a_row(h, counts, max_len, q_unit):
    # equal keys have equal scores: the row is the mean of the values (P in FP16, sums and the mean in FP32)
    c = _cache("i8", 64, max_len, k_scale=1.0)
    c.codes["k"][:] = 3.0
    c.buf["k"].fill_(3)
    qt, _ = to_fp(-q_unit * np.random.default_rng(4).uniform(1.0, 1.5, (sum(counts), 2 * 64)), "bf16")
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy()
    for b, (n, at) in enumerate(zip(counts, starts(counts))):
        v = c.values("v", b)[:, 0]
        for i in range(n):
            seen = v[:LENS[b] - n + i + 1]
            bar = 2.0 ** -10 * np.abs(seen).mean(0) + 2.0 ** -8 * np.abs(seen.mean(0))
            assert np.all(np.abs(got[at + i] - np.tile(seen.mean(0), 2)) <= np.tile(bar, 2)), (b, i)


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
def test_subnormal_queries(h, kind, dh, counts, max_len):
    # BF16 queries of 1e-39 against keys of 1e37: scores of about one
    c = _cache(kind, dh, max_len)
    c.scale["k"][:] = np.float32(5e35) * np.random.default_rng(5).uniform(0.3, 1.0, c.scale["k"].shape)
    _renew(c, "k")
    qt, qx = to_fp(1e-39 * np.random.default_rng(6).standard_normal((sum(counts), 2 * dh)), "bf16")
    assert qx.any()
    _compare(c, _run(h, c, qt, counts, 2, "bf16", scale=20.0), qx, counts, 2, "bf16", scale=20.0)


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("kind,dh", [("i8", 64), ("f8", 128)])
@pytest.mark.parametrize("q_unit", [1e3, 1e5, 1e6, 3e6, 1e7, 4e7, 1e9, 1e12])
def test_large_scores_whose_maximum_comes_late(h, kind, dh, counts, max_len, q_unit):
    # positive scores that grow from page to page, the last tokens' but for one that is larger than all: the maximum moves at many places
    c = _cache(kind, dh, max_len, k_scale=1.0)
    late = [130, 100]
    codes = c.codes["k"]
    for b in range(2):
        for i, pid in enumerate(c.table[b]):
            codes[pid] = BC.to_codes(np.full(codes[pid].shape, 4.0 + 3.0 * min(i, 12)), kind)
        codes[c.table[b][late[b] // 16], :, late[b] % 16] = 112.0
    c.buf["k"].copy_(torch.from_numpy(codes.astype(np.float32)).to(c.buf["k"].dtype))
    qt, _ = to_fp(q_unit * np.random.default_rng(8).uniform(1.0, 1.5, (sum(counts), 2 * dh)), "bf16")
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy()
    for b, (n, at) in enumerate(zip(counts, starts(counts))):
        want = np.tile(c.values("v", b)[late[b], 0], (n, 2))
        sees = LENS[b] - n + np.arange(n) >= late[b]
        assert sees.any() and np.all((np.abs(got[at:at + n] - want) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(want))[sees]), b


@pytest.mark.parametrize("counts,max_len", FORMS)
@pytest.mark.parametrize("kind,dh", [("i8", 128), ("f8", 64)])
def test_rows_of_very_different_size_side_by_side(h, kind, dh, counts, max_len):
    # ordinary rows beside rows a billion times as large, whose largest key is all that counts (where the next is 2^-12 of the scores away)
    c = _cache(kind, dh, max_len)
    rows = sum(counts)
    q = np.random.default_rng(9).standard_normal((rows, 2, dh))
    q[:, 1] *= 10.0 ** (3 * (np.arange(rows) % 4))[:, None]                  # head 1: 1, 1e3, 1e6, 1e9
    qt, qx = to_fp(q.reshape(rows, 2 * dh), "bf16")
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy().reshape(rows, 2, dh)
    want, bar = (x.reshape(rows, 2, dh) for x in _expect(c, qx, counts, 2, dh ** -0.5, rows))
    bar = bar + 2.0 ** -8 * (np.abs(want) + bar)
    assert np.all(np.abs(got - want)[:, 0] <= bar[:, 0])
    sure = 0
    for b, (n, at) in enumerate(zip(counts, starts(counts))):
        k, v = c.values("k", b)[:, 0], c.values("v", b)[:, 0]
        for i in range(n):
            m = LENS[b] - n + i + 1
            s = k[:m] @ qx.reshape(rows, 2, dh)[at + i, 1] * dh ** -0.5
            top, runner = np.sort(s)[-1], np.sort(s)[-2] if m > 1 else -np.inf
            if (at + i) % 4 >= 2 and top - runner > 2.0 ** -12 * np.abs(s).max():
                sure += 1
                one = v[int(np.argmax(s))]
                assert np.all(np.abs(got[at + i, 1] - one) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(one)), (b, i)
    assert sure or rows < 4
