"""GPU parity of hero_block_attention where its work is dealt out differently: row tiles of every size, more sequences than a CTA keeps
in shared memory, more groups than CTAs, nothing to do, maxima and value scales that move, caches beyond four gigabytes, two
streams at once.  Bounds as in test_gpu_block_attention.py."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero
from block_util import Cache, FP, start_tensor, starts, to_fp
from test_gpu_block_attention import _compare, _expect, _q, _run

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


@pytest.mark.parametrize("group,counts", [(4, [6, 1, 0, 5, 3]), (8, [3, 2, 1, 3, 1]), (1, [20, 24, 1, 0, 17]), (1, [32, 25, 3, 9, 31]), (5, [6, 5, 4, 1, 2]),
                                          (33, [1, 1, 1, 1, 1]), (40, [2, 1, 2, 0, 1])])
@pytest.mark.parametrize("dh,kind", [(64, "f8"), (128, "i8")])
def test_row_tiles_of_every_size(h, group, counts, dh, kind):
    lens = [700, 40, 9, 1025, 333]
    c = Cache(80 + group, kind, 32, 2, dh, lens, max_len=1500)
    qt, qx = _q(1, sum(counts) + 1, 2 * group * dh, "bf16")
    _compare(c, _run(h, c, qt, counts, 2 * group, "bf16"), qx, counts, 2 * group, "bf16")


@pytest.mark.parametrize("layout", ["nhd", "padded"])
@pytest.mark.parametrize("page", [16, 128])
def test_prompts_of_several_row_tiles_in_any_layout(h, layout, page):
    counts, lens = [300, 129, 1, 0, 256], [300, 400, 77, 5, 1000]
    c = Cache(90 + page, "i8", page, 2, 128, lens, max_len=1200, layout=layout)
    qt, qx = _q(2, sum(counts) + 2, 4 * 128, "f16")
    _compare(c, _run(h, c, qt, counts, 4, "f16"), qx, counts, 4, "f16")


def test_more_sequences_and_groups_than_are_kept_or_resident(h):
    B, nkv, dh = 700, 2, 64
    g = np.random.default_rng(3)
    lens = [int(x) for x in g.integers(0, 60, B)]
    lens[5], lens[300], lens[699] = 900, 640, 513
    counts = [int(x) for x in g.integers(0, 3, B)]
    c = Cache(95, "i8", 16, nkv, dh, lens, max_len=1000)
    qt, qx = _q(3, sum(counts), 2 * nkv * dh, "f16")
    _compare(c, _run(h, c, qt, counts, 2 * nkv, "f16"), qx, counts, 2 * nkv, "f16")


@pytest.mark.parametrize("max_rows,max_len", [(1, 100), (1, 9000), (64, 9000)])
def test_sequences_without_rows_or_tokens(h, max_rows, max_len):
    # no rows at all: nothing is written; rows without a token: zeros, whatever the kernel
    c = Cache(96, "f8", 64, 2, 64, [0, 10, 0], max_len=max_len)
    qt, _ = _q(4, 3, 4 * 64, "bf16")
    out = _run(h, c, qt, [0, 0, 0], 4, "bf16", max_rows=max_rows)
    assert torch.all(out == 7.0)
    c.set_lens([0, 0, 0])
    out = _run(h, c, qt, [1, 1, 1], 4, "bf16", max_rows=max_rows)
    assert torch.all(out == 0)


@pytest.mark.parametrize("counts", [[1, 1], [5, 2], [100, 60]])
@pytest.mark.parametrize("kind", ["i8", "f8"])
def test_maxima_and_value_scales_that_keep_moving(h, counts, kind):
    # every page's keys are about 1.5 times as large as the page's before, so a row's largest score moves up again and again; the value
    # scales rise by a factor of 3 a page.  Probabilities below FP16's normal range are off by half of its smallest step, 2^-25, under a factor
    # of at least 2^8 by which P is formed, in units of the largest value scale: 2^-33 of the largest |v| per key.
    lens = [500, 380]
    c = Cache(97, kind, 32, 1, 64, lens)
    for b in range(2):
        for i, pid in enumerate(c.table[b]):
            c.scale["k"][pid] = 0.002 * 1.5 ** i
            c.scale["v"][pid] = 1e-4 * 3.0 ** i
    for x in "kv":
        c.scale_t[x].copy_(torch.from_numpy(c.scale[x]))
    rows = sum(counts)
    qt, qx = _q(5, rows, 4 * 64, "bf16")
    out = _run(h, c, qt, counts, 4, "bf16")
    want, bar = _expect(c, qx, counts, 4, 64 ** -0.5, rows)
    reach = np.concatenate([np.full(n, np.abs(c.values("v", b)).max()) for b, n in enumerate(counts)])[:, None]
    bar = bar + 500 * 2.0 ** -33 * reach
    bar = bar + torch.finfo(torch.bfloat16).eps / 2 * (np.abs(want) + bar)
    got = out.double().cpu().numpy()
    assert np.all(np.abs(got - want) <= bar), np.max(np.abs(got - want) / bar)


def test_value_scales_that_begin_with_zero(h):
    # pages of zeros first (scale 0), loud pages behind them: what was summed under scale 0 counts nothing
    for counts in ([1], [80]):
        c = Cache(98, "i8", 16, 1, 128, [200])
        for i, pid in enumerate(c.table[0]):
            if i < 9:
                c.scale["v"][pid] = 0
        c.scale_t["v"].copy_(torch.from_numpy(c.scale["v"]))
        qt, qx = _q(6, counts[0], 2 * 128, "f16")
        _compare(c, _run(h, c, qt, counts, 2, "f16"), qx, counts, 2, "f16")


def test_attention_beyond_four_gigabytes(h):
    page, nkv, dh = 128, 8, 128
    n = int(4.6e9 // (page * nkv * dh))
    buf = torch.zeros(n, nkv, page, dh, dtype=torch.int8, device="cuda")
    scale = torch.zeros(n, nkv, device="cuda")
    table = torch.tensor([[n - 1, 0], [n // 2, n - 2]], dtype=torch.int32, device="cuda")
    small = Cache(99, "i8", page, nkv, dh, [200, 130], max_len=256)
    for b in range(2):
        for i in range(2):
            buf[int(table[b, i])] = small.buf["k"][int(small.table[b, i])]
            scale[int(table[b, i])] = small.scale_t["k"][int(small.table[b, i])]
    small.codes["v"], small.scale["v"] = small.codes["k"], small.scale["k"]          # one buffer for both
    small.desc = hero.block_cache(buf, buf, scale, scale, table, small.lens_t, 256)
    for counts in ([1, 1], [60, 40]):
        qt, qx = _q(7, sum(counts), 2 * nkv * dh, "bf16")
        _compare(small, _run(h, small, qt, counts, 2 * nkv, "bf16"), qx, counts, 2 * nkv, "bf16")


def test_two_streams_with_a_workspace_each(h):
    cs = [Cache(100 + i, "i8", 64, 2, 128, [5000, 900, 3000], max_len=6000) for i in range(2)]
    qs = [_q(8 + i, 3, 8 * 128, "bf16") for i in range(2)]
    want = [_run(h, c, q[0], [1] * 3, 8, "bf16") for c, q in zip(cs, qs)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = [torch.zeros_like(w) for w in want]
    wss = [torch.empty(h.hero_block_attention_workspace_bytes(c.desc, 8, 3, 1), dtype=torch.uint8, device="cuda") for c in cs]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, s in enumerate(streams):
            h.hero_block_attention(cs[i].desc, hero.tensor(qs[i][0]), hero.tensor(outs[i]), 8, workspace=wss[i], stream=s)
    torch.cuda.synchronize()
    h.check()
    for o, w in zip(outs, want):
        assert torch.equal(o, w)


def test_a_prompt_and_its_steps_agree(h):
    # a prompt is appended and attended to in one call; the same tokens one by one, each appended and attended to, on a cache of their own,
    # see scales that grew differently: both against the oracle on the codes that the device holds
    nq, nkv, dh, n = 4, 2, 64, 50
    g = np.random.default_rng(11)
    kt, _ = to_fp(g.standard_normal((n, nkv * dh)), "f16")
    vt, _ = to_fp(g.standard_normal((n, nkv * dh)), "f16")
    qt, qx = _q(12, n, nq * dh, "f16")
    c = Cache(101, "i8", 16, nkv, dh, [n], max_len=64)
    s = start_tensor([n])
    h.hero_block_cache_append(c.desc, hero.tensor(kt), hero.tensor(vt), row_start=s, max_rows=n)
    out = _run(h, c, qt, [n], nq, "f16")
    for x in "kv":
        c.codes[x], c.scale[x] = c.device_codes(x), c.scale_t[x].cpu().numpy()
    _compare(c, out, qx, [n], nq, "f16")
    d = Cache(102, "i8", 16, nkv, dh, [n], max_len=64)
    for i in range(n):
        d.set_lens([i + 1])
        h.hero_block_cache_append(d.desc, hero.tensor(kt[i:i + 1]), hero.tensor(vt[i:i + 1]))
        step = _run(h, d, qt[i:i + 1], [1], nq, "f16")
        for x in "kv":
            d.codes[x], d.scale[x] = d.device_codes(x), d.scale_t[x].cpu().numpy()
        _compare(d, step, qx[i:i + 1], [1], nq, "f16")


@pytest.mark.parametrize("counts", [[1, 1, 1], [20, 5, 60]])
def test_what_is_not_finite_in_a_query_stays_in_its_row(h, counts):
    c = Cache(104, "i8", 16, 2, 64, [90, 33, 70])
    rows = sum(counts) + 2
    qt, qx = _q(13, rows, 4 * 64, "bf16")
    want = _run(h, c, qt, counts, 4, "bf16")
    bad = qt.clone()
    bad[0, 64:128] = float("nan")                                            # head 1 of the first row
    bad[counts[0], 5] = float("inf")                                         # head 0 of the second sequence's first row
    bad[-2:] = float("nan")                                                  # rows of nobody
    got = _run(h, c, bad, counts, 4, "bf16")
    assert torch.all(torch.isnan(got[0, 64:128]))
    keep = torch.ones_like(got, dtype=torch.bool)
    keep[0, 64:128] = keep[counts[0], :64] = False
    assert torch.equal(got[keep], want[keep])


def test_tensors_of_another_device_are_refused(h):
    # one GPU is visible: the handle is told that it belongs to another one
    c = Cache(105, "i8", 16, 1, 64, [5, 5])
    q = hero.tensor(torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda"))
    pinned = hero.host_tensor(torch.zeros(2, 64, dtype=torch.bfloat16))
    with pytest.raises(hero.HeroError, match="device"):
        h.hero_block_attention(c.desc, pinned, q, 1)
    with pytest.raises(hero.HeroError, match="device"):
        h.hero_block_cache_append(c.desc, q, pinned)
    own = h._device
    try:
        h._device = own + 1
        with pytest.raises(hero.HeroError, match="device"):
            h.hero_block_attention(c.desc, q, q, 1)
        with pytest.raises(hero.HeroError, match="device"):
            h.hero_qk_norm_rope(q, None, q, None, 1, 0)
    finally:
        h._device = own


def test_binding_refusals(h):
    c = Cache(103, "i8", 16, 1, 64, [5, 5])
    q = hero.tensor(torch.zeros(2, 64, dtype=torch.bfloat16, device="cuda"))
    ok = start_tensor([1, 1])
    for kw in (dict(row_start=ok[:2]), dict(row_start=ok.long()), dict(row_start=ok.cpu()), dict(workspace=torch.zeros(64, dtype=torch.float32, device="cuda")),
               dict(workspace=torch.zeros(64, dtype=torch.uint8))):
        with pytest.raises(hero.HeroError):
            h.hero_block_attention(c.desc, q, q, 1, **kw)
    k = c.buf["k"]
    with pytest.raises(hero.HeroError):
        hero.block_cache(k, k[:, :, :8], c.scale_t["k"], c.scale_t["v"], c.table_t, c.lens_t, 5)
    with pytest.raises(hero.HeroError):
        hero.block_cache(k, k, c.scale_t["k"].double(), c.scale_t["v"], c.table_t, c.lens_t, 5)
    with pytest.raises(hero.HeroError):
        hero.block_cache(k, k, c.scale_t["k"], c.scale_t["v"], c.table_t, c.lens_t[:1], 5)
    with pytest.raises(hero.HeroError):
        hero.block_cache(k, k, c.scale_t["k"], c.scale_t["v"], c.table_t.cpu(), c.lens_t, 5)


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("counts,lens,group,nkv,dh,page,max_len,layout", [
    ([40], [5000], 4, 2, 128, 64, 5000, "hnd"),                  # ten parts of a group
    ([70, 33], [2100, 150], 1, 1, 64, 16, 2100, "nhd"),          # fewer tiles of keys than parts
    ([300, 0, 3], [3001, 2000, 3], 2, 2, 128, 32, 3100, "padded"),   # several row tiles, the rows of one end inside the last part
    ([50, 40], [20, 1281], 3, 2, 64, 128, 1400, "hnd"),          # rows from before the first token: zeros
])
def test_few_groups_whose_keys_are_split(h, kind, counts, lens, group, nkv, dh, page, max_len, layout):
    c = Cache(105 + len(counts) + page, kind, page, nkv, dh, lens, max_len=max_len, layout=layout)
    nq = group * nkv
    qt, qx = _q(15, sum(counts) + 2, nq * dh, "bf16")
    assert h.hero_block_attention_workspace_bytes(c.desc, nq, qt.shape[0], max(counts)) > 0
    out = _run(h, c, qt, counts, nq, "bf16")
    _compare(c, out, qx, counts, nq, "bf16")
    assert torch.equal(out, _run(h, c, qt, counts, nq, "bf16"))


@pytest.mark.parametrize("kind", ["i8", "f8"])
def test_split_keys_with_maxima_and_value_scales_that_move(h, kind):
    # bound as in test_maxima_and_value_scales_that_keep_moving: 2^-33 of the largest |v| per key for probabilities below FP16's normal range
    counts, lens, page, nkv, dh = [64], [2600], 32, 1, 128
    c = Cache(120, kind, page, nkv, dh, lens)
    g = np.random.default_rng(16)
    for x, lo, hi in (("k", -6, 3), ("v", -20, 8)):
        c.scale[x] = (c.scale[x] * np.exp2(g.uniform(lo, hi, c.scale[x].shape))).astype(np.float32)
        c.scale_t[x].copy_(torch.from_numpy(c.scale[x]))
    qt, qx = _q(17, 64, 2 * dh, "bf16", size=2.0)
    got = _run(h, c, qt, counts, 2, "bf16").double().cpu().numpy()
    want, bar = _expect(c, qx, counts, 2, dh ** -0.5, 64)
    bar = bar + lens[0] * 2.0 ** -33 * np.abs(c.values("v", 0)).max()
    bar = bar + torch.finfo(torch.bfloat16).eps / 2 * (np.abs(want) + bar)
    assert np.all(np.abs(got - want) <= bar), np.max(np.abs(got - want) / bar)


def test_split_keys_not_finite_queries_and_eight_bit_outputs(h):
    counts, lens, nkv, dh, nq = [60, 45], [2000, 1100], 2, 64, 4
    c = Cache(121, "i8", 16, nkv, dh, lens)
    rows = sum(counts)
    qt, qx = _q(18, rows, nq * dh, "bf16")
    want, bar = _expect(c, qx, counts, nq, dh ** -0.5, rows)
    bad = qt.clone()
    bad[7, dh:2 * dh] = float("nan")
    bad[60, 5] = float("inf")
    out = _run(h, c, bad, counts, nq, "bf16")
    assert torch.all(torch.isnan(out[7, dh:2 * dh]))
    keep = np.ones(want.shape, dtype=bool)
    keep[7, dh:2 * dh] = keep[60, :dh] = False
    near = bar + torch.finfo(torch.bfloat16).eps / 2 * (np.abs(want) + bar)
    assert np.all(np.abs(out.double().cpu().numpy() - want)[keep] <= near[keep])
    step = np.float32(np.abs(want).max() / 127 * 0.9)                        # some saturate
    codes = torch.zeros(rows, nq * dh, dtype=torch.int8, device="cuda")
    _run(h, c, qt, counts, nq, "bf16", out=codes, gran="sq", out_scale=torch.tensor([step], device="cuda"))
    y, d = want / step, bar / step * 1.01 + 1e-5
    got = codes.double().cpu().numpy()
    assert np.all((got >= BC.to_codes(y - d, "i8")) & (got <= BC.to_codes(y + d, "i8")))   # rounding is monotonic


def test_split_keys_captured_and_replayed_at_other_lengths(h):
    counts, nkv, dh, nq = [48], 2, 64, 4
    c = Cache(122, "i8", 64, nkv, dh, [4000])
    qt, qx = _q(19, 48, nq * dh, "f16")
    out = torch.full((48, nq * dh), 7.0, dtype=torch.float16, device="cuda")
    s = start_tensor(counts)
    ws = torch.full((h.hero_block_attention_workspace_bytes(c.desc, nq, 48, 48),), 0xff, dtype=torch.uint8, device="cuda")

    def call():
        h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out), nq, row_start=s, max_rows=48, workspace=ws)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            call()
    torch.cuda.synchronize()
    for n in (4000, 130, 60, 3333):
        c.set_lens([n])
        graph.replay()
        torch.cuda.synchronize()
        h.check()
        _compare(c, out, qx, counts, nq, "f16")
