"""GPU parity: hero_block_cache_append and hero_block_cache_read against the oracle, to the bit (the definition is in FP32 with
correctly rounded division, so codes, scales and read-back values have one right answer)."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero
from block_util import Cache, FP, start_tensor, starts, to_fp

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def _rows(seed, rows, width, fp, loud=True):
    g = np.random.default_rng(seed)
    x = g.standard_normal((rows, width)) * np.exp(g.standard_normal((rows, 1)))
    if loud:
        x[:, g.integers(0, width, max(1, width // 40))] *= 8
    return to_fp(x, fp)


def _append_and_compare(h, c, counts, kx, vx, kt, vt, pad=0):
    """Runs the append on the device and in the oracle; compares every code and scale of the pool."""
    s = None if counts is None else start_tensor(counts)
    n = counts if counts is not None else [1] * len(c.lens)
    h.hero_block_cache_append(c.desc, hero.tensor(kt), hero.tensor(vt), row_start=s, max_rows=max(max(n), 1))
    h.check()
    for x, data in (("k", kx), ("v", vx)):
        codes, scale = BC.append(c.codes[x], c.scale[x], c.table, c.lens, n, starts(n), data, c.page, c.kind)
        got_s, got = c.scale_t[x].cpu().numpy(), c.device_codes(x)
        assert np.array_equal(got_s, scale), "%s: %d scales differ" % (x, np.sum(got_s != scale))
        assert np.array_equal(got, codes), "%s: %d codes differ" % (x, np.sum(got != codes))
        c.codes[x], c.scale[x] = codes, scale


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("page,dh,layout", [(16, 64, "hnd"), (32, 128, "nhd"), (64, 64, "padded"), (128, 128, "hnd"), (16, 128, "padded"), (128, 64, "nhd"),
                                            (32, 64, "hnd"), (64, 128, "hnd")])
def test_append_ragged_prompts_to_the_bit(h, kind, fp, page, dh, layout):
    nkv = 3
    counts = [1, 0, page, 2 * page + 5, 7, 3 * page]
    held = [page - 1, 9, 0, page // 2, 3 * page, page]         # the page that is begun, filled to the border, left half full
    lens = [a + n for a, n in zip(held, counts)]
    c = Cache(5 + page + dh, kind, page, nkv, dh, lens, layout=layout)
    rows = sum(counts) + 4                                     # rows behind the last sequence belong to nobody
    kt, kx = _rows(1, rows, nkv * dh, fp)
    vt, vx = _rows(2, rows, nkv * dh, fp)
    _append_and_compare(h, c, counts, kx, vx, kt, vt)


@pytest.mark.parametrize("kind", ["i8", "f8"])
def test_append_token_by_token_to_the_bit(h, kind):
    # forty decode steps over page borders: scales grow, earlier tokens of the page are quantised again
    page, nkv, dh, B = 16, 2, 64, 3
    c = Cache(3, kind, page, nkv, dh, [1, 14, 30], max_len=80)
    for step in range(40):
        kt, kx = _rows(100 + step, B, nkv * dh, "bf16")
        vt, vx = _rows(200 + step, B, nkv * dh, "bf16")
        _append_and_compare(h, c, None, kx, vx, kt, vt)
        c.set_lens([n + 1 for n in c.lens])


def test_append_from_strided_rows(h):
    # k and v are the last two thirds of a QKV row block
    nkv, dh, page = 2, 128, 32
    c = Cache(8, "i8", page, nkv, dh, [40, 33])
    t, x = _rows(4, 60, 3 * nkv * dh, "bf16")
    w = nkv * dh
    _append_and_compare(h, c, [40, 20], x[:, w:2 * w], x[:, 2 * w:], t[:, w:2 * w], t[:, 2 * w:])


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("fp", ["f16", "bf16"])
def test_append_values_that_go_wrong(h, kind, fp):
    # zeros, subnormals, the type's largest, NaN and infinities, ties of the quotient, scales far below the fast division's range
    page, nkv, dh = 16, 1, 64
    counts = [16] * 8
    c = Cache(9, kind, page, nkv, dh, counts)
    g = np.random.default_rng(0)
    big = float(torch.finfo(FP[fp]).max)
    tiny = float(torch.finfo(FP[fp]).smallest_normal)
    x = g.standard_normal((16 * 8, dh))
    x[0:16] = 0
    x[16:32] *= tiny                                            # subnormal quotients of a tiny scale
    x[32:48] = big * np.sign(x[32:48])
    x[48:64, ::7] = np.nan
    x[64:80, 3], x[64:80, 5] = np.inf, -np.inf
    x[80:96] = np.nan
    x[96:112] = g.integers(-254, 255, (16, dh)) / 2.0           # scale 1 exactly after the next line: halves are ties
    x[96, 0] = 127.0
    x[96:112] = np.clip(x[96:112], -127, 127)
    x[112:128] = 0
    x[112, 1], x[113, 2] = np.inf, np.nan                       # an infinity over a zero scale
    t, xr = to_fp(x, fp)
    _append_and_compare(h, c, counts, xr, xr, t, t)
    if fp == "bf16":                                            # scales of 1e-37 .. 1e-39: the plain division
        x2 = g.standard_normal((128, dh)) * 10.0 ** -(36 + np.arange(128) // 16)[:, None]
        t, xr = to_fp(x2, fp)
        c2 = Cache(10, kind, page, nkv, dh, counts)
        _append_and_compare(h, c2, counts, xr, xr, t, t)


def test_quotients_are_correctly_rounded(h):
    # a million quotients of one scale each page: with scale = absmax / 127 the codes of every FP16 value below it
    page, nkv, dh = 128, 8, 128
    all16 = torch.arange(0, 0x7c00, dtype=torch.int16).view(torch.float16)
    g = torch.Generator().manual_seed(4)
    for seed in range(3):
        pick = all16[torch.randint(0, all16.numel(), (page * 4, nkv * dh), generator=g)].clone()
        x = pick * torch.where(torch.rand(pick.shape, generator=g) < 0.5, 1, -1).half()
        c = Cache(20 + seed, "i8", page, nkv, dh, [page] * 4)
        xr = x.double().numpy()
        _append_and_compare(h, c, [page] * 4, xr, xr, x.cuda(), x.cuda())


def test_append_leaves_other_pages_and_slots_alone_and_refuses_bad_pages(h):
    page, nkv, dh = 16, 2, 64
    c = Cache(11, "i8", page, nkv, dh, [20, 20])
    kt, kx = _rows(1, 40, nkv * dh, "f16")
    bad = c.table.copy()
    bad[0, 1], bad[1, 0] = c.n_pages, -3
    c.table_t.copy_(torch.from_numpy(bad))
    h.hero_block_cache_append(c.desc, hero.tensor(kt), hero.tensor(kt), row_start=start_tensor([20, 20]), max_rows=20)
    with pytest.raises(hero.HeroError) as e:
        h.check()
    assert e.value.status == hero.ERR_INVALID_ARG and "page" in str(e.value)
    h.check()                                                  # reported once
    codes, scale = BC.append(c.codes["k"], c.scale["k"], bad, c.lens, [20, 20], [0, 20], kx, page, "i8")
    assert np.array_equal(c.device_codes("k"), codes) and np.array_equal(c.scale_t["k"].cpu().numpy(), scale)


def test_append_cuts_bad_row_ranges_and_lengths(h):
    page, nkv, dh = 16, 1, 64
    kt, kx = _rows(1, 10, nkv * dh, "f16")
    for start, max_rows, lens, eff in (([0, 5, 99], 10, [5, 5], ([0, 5], [5, 5])),           # beyond the matrix
                                       ([0, 7, 3], 10, [7, 5], ([0, 7], [7, 0])),            # decreasing
                                       ([0, 6, 10], 4, [6, 4], ([0, 6], [4, 4])),            # longer than max_rows
                                       ([-4, 2, 4], 10, [2, 2], ([0, 2], [2, 2]))):          # negative
        c = Cache(12, "i8", page, nkv, dh, lens)
        h.hero_block_cache_append(c.desc, hero.tensor(kt), hero.tensor(kt), row_start=torch.tensor(start, dtype=torch.int32, device="cuda"), max_rows=max_rows)
        with pytest.raises(hero.HeroError, match="row range"):
            h.check()
        codes, _ = BC.append(c.codes["k"], c.scale["k"], c.table, c.lens, eff[1], eff[0], kx, page, "i8")
        assert np.array_equal(c.device_codes("k"), codes), start
    # more rows than the sequence holds: the first ones have no token; a length beyond max_len or below 0 is cut
    c = Cache(13, "i8", page, nkv, dh, [3, 4], max_len=32)
    c.lens_t.copy_(torch.tensor([3, -7], dtype=torch.int32))
    h.hero_block_cache_append(c.desc, hero.tensor(kt), hero.tensor(kt), row_start=start_tensor([5, 5]), max_rows=5)
    h.check()
    codes, _ = BC.append(c.codes["k"], c.scale["k"], c.table, [3, 0], [5, 5], [0, 5], kx, page, "i8")
    assert np.array_equal(c.device_codes("k"), codes)


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("page,dh,nkv,layout", [(16, 64, 1, "hnd"), (32, 128, 5, "nhd"), (128, 128, 2, "padded"), (64, 64, 20, "hnd")])
def test_read_to_the_bit(h, kind, fp, page, dh, nkv, layout):
    lens, counts = [1, 0, 200, 77, 4], [1, 0, 200, 13, 6]       # the last one has two rows without a token
    c = Cache(30 + nkv, kind, page, nkv, dh, lens, layout=layout)
    rows = sum(counts) + 3
    out = {x: torch.full((rows, nkv * dh), 7.0, dtype=FP[fp], device="cuda") for x in "kv"}
    h.hero_block_cache_read(c.desc, hero.tensor(out["k"]), hero.tensor(out["v"]), row_start=start_tensor(counts), max_rows=200)
    h.check()
    for x in "kv":
        want = np.full((rows, nkv * dh), 7.0)
        for b, (n, m, s) in enumerate(zip(lens, counts, starts(counts))):
            v = (c.codes[x].astype(np.float32) * c.scale[x][:, :, None, None])       # FP32, then one rounding
            y = BC.tokens(v.astype(np.float64), np.ones_like(c.scale[x]), c.table[b], n, page).reshape(n, nkv * dh)
            y = np.concatenate([np.zeros((max(0, m - n), nkv * dh)), y[max(0, n - m):]])
            want[s:s + m] = torch.from_numpy(y.astype(np.float32)).to(FP[fp]).double().numpy() if m else want[s:s + m]
        assert np.array_equal(out[x].double().cpu().numpy(), want), x


def test_read_one_of_the_two_one_row_each_and_into_wider_rows(h):
    c = Cache(40, "i8", 32, 2, 64, [5, 64, 33])
    wide = torch.zeros(3, 2 * 128, dtype=torch.bfloat16, device="cuda")
    h.hero_block_cache_read(c.desc, None, hero.tensor(wide[:, 128:]))
    h.check()
    for b, n in enumerate(c.lens):
        want = torch.from_numpy(c.values("v", b)[n - 1].reshape(-1)).float().bfloat16()
        assert torch.equal(wide[b, 128:].cpu(), want)
    assert torch.all(wide[:, :128] == 0)


def test_read_clamps_and_reports_bad_pages(h):
    c = Cache(41, "i8", 16, 1, 64, [32])
    c.table_t.copy_(torch.tensor([[c.n_pages + 5, int(c.table[0, 1])]], dtype=torch.int32))
    out = torch.zeros(32, 64, dtype=torch.float16, device="cuda")
    h.hero_block_cache_read(c.desc, hero.tensor(out), None, row_start=start_tensor([32]), max_rows=32)
    with pytest.raises(hero.HeroError, match="page"):
        h.check()
    v = c.codes["k"] * c.scale["k"].astype(np.float64)[:, :, None, None]
    want = torch.from_numpy(np.concatenate([v[c.n_pages - 1, 0], v[c.table[0, 1], 0]]).astype(np.float32)).half()
    assert torch.equal(out.cpu(), want)


def test_a_cache_beyond_four_gigabytes(h):
    # pages whose offset passes 2^32 bytes: the first, one in the middle and the last of a 4.6 GB pool (k and v share one buffer,
    # and both are given the same rows)
    page, nkv, dh = 128, 8, 128
    n = int(4.6e9 // (page * nkv * dh))
    buf = torch.zeros(n, nkv, page, dh, dtype=torch.int8, device="cuda")
    scale = torch.zeros(n, nkv, device="cuda")
    table = torch.tensor([[n - 1, 0], [n // 2, n - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([200, 130], dtype=torch.int32, device="cuda")
    kt, kx = _rows(1, 330, nkv * dh, "bf16")
    d = hero.block_cache(buf, buf, scale, scale, table, lens, 256)
    h.hero_block_cache_append(d, hero.tensor(kt), hero.tensor(kt), row_start=start_tensor([200, 130]), max_rows=200)
    out = torch.zeros(330, nkv * dh, dtype=torch.bfloat16, device="cuda")
    h.hero_block_cache_read(d, hero.tensor(out), None, row_start=start_tensor([200, 130]), max_rows=200)
    h.check()
    codes, sc = BC.append(np.zeros((4, nkv, page, dh)), np.zeros((4, nkv)), [[3, 0], [1, 2]], [200, 130], [200, 130], [0, 200], kx, page, "i8")
    want = np.concatenate([BC.tokens(codes, sc, [3, 0], 200, page), BC.tokens(codes, sc, [1, 2], 130, page)]).reshape(330, -1)
    assert torch.equal(out.cpu(), torch.from_numpy(want.astype(np.float32)).bfloat16())
