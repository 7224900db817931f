"""GPU parity: hero_block_attention against the oracle in fp64 on the values that the cache's codes stand for.

Bound of one output element, with P the exact probabilities and mass = sum P |v|: a score is a sum of dh exact products in
FP32 (each addition, tensor core included, counted as 2^-23 of the sum of magnitudes), times two scale factors, then 2^x to a
few units: an exponent error d of at most (dh + 4) 2^-23 * size, size the largest sum |q_c k_c| scale of the row; a probability is
off by exp(2 d) - 1 (numerator and sum), by half a step of FP16 (2^-11; below 2^-14 of the row's largest an absolute 2^-25 of the
largest |v| in reach), and by the FP32 sums over L keys (2^-23 L).  The result is rounded once to its type."""
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


def _expect(c, qx, counts, nq, scale, rows):
    """(want, bound without the output's rounding), [rows, nq * dh]; rows of nobody: NaN."""
    dh, group = c.dh, nq // c.nkv
    want, bar = np.full((rows, nq * dh), np.nan), np.zeros((rows, nq * dh))
    for b, (n, at) in enumerate(zip(counts, starts(counts))):
        if n == 0:
            continue
        k, v = c.values("k", b), c.values("v", b)
        L = max(c.lens[b], 0)
        o, mass, size = BC.attention(qx[at:at + n].reshape(n, nq, dh), k, v, group, scale)
        d = (dh + 4) * 2.0 ** -23 * size[..., None]
        reach = np.repeat(np.abs(v).max((0, 2)) if L else np.zeros(c.nkv), group)[None, :, None]
        e = mass * (np.expm1(2 * d) + 2.0 ** -11 + 2.0 ** -23 * max(L, 1) + 2.0 ** -20) + L * 2.0 ** -25 * reach * 2.0 ** -11
        want[at:at + n], bar[at:at + n] = o.reshape(n, -1), e.reshape(n, -1)
    return want, bar


def _run(h, c, qt, counts, nq, fp, scale=0.0, out=None, gran="none", out_scale=None, max_rows=None):
    out = torch.full((qt.shape[0], nq * c.dh), 7.0, dtype=FP[fp], device="cuda") if out is None else out
    most = max_rows or max(max(counts), 1)
    s = start_tensor(counts)
    n = h.hero_block_attention_workspace_bytes(c.desc, nq, qt.shape[0], most)
    ws = torch.full((n,), 0xff, dtype=torch.uint8, device="cuda")          # NaN patterns: nothing may depend on what it held
    h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out, gran, out_scale), nq, row_start=s, max_rows=most, scale=scale, workspace=ws)
    h.check()
    return out


def _compare(c, out, qx, counts, nq, fp, scale=None):
    want, bar = _expect(c, qx, counts, nq, scale or c.dh ** -0.5, qx.shape[0])
    got = out.double().cpu().numpy()
    live = ~np.isnan(want[:, 0])
    assert np.all(got[~live] == 7.0)                                       # rows of nobody are left as they were
    want, bar, got = want[live], bar[live], got[live]
    bar = bar + torch.finfo(FP[fp]).eps / 2 * (np.abs(want) + bar) + (2.0 ** -25 if fp == "f16" else 0)
    bad = ~(np.abs(got - want) <= bar)
    assert not bad.any(), "%d of %d outside, worst %.3g of the bound" % (bad.sum(), bad.size, np.nanmax(np.abs(got - want) / bar))


def _q(seed, rows, width, fp, size=1.0):
    return to_fp(np.random.default_rng(seed).standard_normal((rows, width)) * size, fp)


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("fp", ["f16", "bf16"])
@pytest.mark.parametrize("page,dh,nkv,group,layout", [
    (16, 64, 2, 1, "hnd"), (16, 128, 1, 4, "padded"), (32, 128, 2, 8, "nhd"), (64, 64, 3, 3, "hnd"), (128, 128, 1, 5, "hnd"), (128, 64, 1, 16, "padded"),
    (64, 128, 1, 12, "nhd")])
def test_one_token_at_odd_lengths(h, kind, fp, page, dh, nkv, group, layout):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 300, 0, 511]
    c = Cache(page + dh + group, kind, page, nkv, dh, lens, layout=layout)
    counts = [1] * len(lens)
    qt, qx = _q(1, len(lens) + 2, nkv * group * dh, fp)
    out = _run(h, c, qt, counts, nkv * group, fp)
    _compare(c, out, qx, counts, nkv * group, fp)
    assert torch.all(out[11] == 0)                                          # a sequence without tokens


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("page,dh,nkv,group,fp", [(16, 64, 2, 1, "f16"), (64, 128, 2, 4, "bf16"), (128, 128, 1, 7, "f16"), (32, 64, 1, 8, "bf16"), (64, 128, 1, 3, "f16")])
def test_several_rows_per_sequence(h, kind, page, dh, nkv, group, fp):
    # drafts and prompt pieces: causal inside the rows, ragged, some sequences without rows, one with more rows than tokens
    counts = [5, 1, 0, 9, 17, 33, 4, 70, 2, 130]
    lens = [5, 40, 77, 9, 18, 200, 2, 300, 129, 131]
    c = Cache(7 + page, kind, page, nkv, dh, lens)
    rows = sum(counts) + 1
    qt, qx = _q(2, rows, nkv * group * dh, fp)
    out = _run(h, c, qt, counts, nkv * group, fp)
    _compare(c, out, qx, counts, nkv * group, fp)
    at = starts(counts)[6]
    assert torch.all(out[at:at + 2] == 0)                                   # the two rows before the first token


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("dh", [64, 128])
def test_a_long_axis_with_few_rows(h, kind, dh):
    # thousands of keys for one sequence beside short ones: the long axis is split and joined
    lens = [9000, 1, 4097, 40]
    c = Cache(50, kind, 64, 1, dh, lens, max_len=20000)
    qt, qx = _q(3, 4, 4 * dh, "f16")
    _compare(c, _run(h, c, qt, [1] * 4, 4, "f16"), qx, [1] * 4, 4, "f16")
    counts = [3, 1, 2, 2]
    qt, qx = _q(4, 8, 4 * dh, "bf16")
    _compare(c, _run(h, c, qt, counts, 4, "bf16"), qx, counts, 4, "bf16")


def test_scores_far_apart_and_scales_of_very_different_size(h):
    # one key outweighs all others, or all weigh the same; page scales spread over twelve orders of magnitude
    c = Cache(60, "i8", 16, 1, 64, [200, 200, 333], k_unit=1.5 / 40)
    g = np.random.default_rng(1)
    for x, lo, hi in (("v", -9, 3), ("k", -3, 0)):
        c.scale[x] = (c.scale[x] * 10.0 ** g.uniform(lo, hi, c.scale[x].shape)).astype(np.float32)
        c.scale_t[x].copy_(torch.from_numpy(c.scale[x]))
    qt, qx = _q(5, 3, 8 * 64, "bf16", size=20.0)
    _compare(c, _run(h, c, qt, [1] * 3, 8, "bf16"), qx, [1] * 3, 8, "bf16")
    qt, qx = to_fp(np.zeros((3, 8 * 64)), "f16")
    _compare(c, _run(h, c, qt, [1] * 3, 8, "f16"), qx, [1] * 3, 8, "f16")
    c.scale["k"][:], c.scale["v"][::2] = 0, 0                                # pages of zeros
    for x in "kv":
        c.scale_t[x].copy_(torch.from_numpy(c.scale[x]))
    qt, qx = _q(6, 3, 8 * 64, "f16")
    _compare(c, _run(h, c, qt, [1] * 3, 8, "f16"), qx, [1] * 3, 8, "f16")


def test_queries_beyond_the_range_of_fp16(h):
    # BF16 queries of 1e20 and of 1e-20 in one call: a row's scale is its own
    c = Cache(61, "i8", 64, 1, 128, [100, 100])
    g = np.random.default_rng(2)
    q = g.standard_normal((2, 128))
    q[0] *= 1e20
    q[1] *= 1e-20
    qt, qx = to_fp(q, "bf16")
    _compare(c, _run(h, c, qt, [1, 1], 1, "bf16", scale=1e-21), qx, [1, 1], 1, "bf16", scale=1e-21)


@pytest.mark.parametrize("counts", [[1, 1, 1], [2, 40, 70]])
def test_what_lies_behind_the_end_of_a_sequence_has_no_effect(h, counts):
    # NaN codes (e4m3 has them) and NaN scales in slots and pages that no row may see
    lens = [70, 40, 129]
    a, b = (Cache(62, "f8", 64, 2, 64, lens, max_len=256) for _ in range(2))
    for x in "kv":
        raw = b.buf[x].view(torch.uint8)
        for s, n in enumerate(lens):
            for pi in range(256 // 64):
                first = min(max(n - pi * 64, 0), 64)
                raw[int(b.table[s, pi]), :, first:] = 0x7f
                if first == 0:
                    b.scale_t[x][int(b.table[s, pi])] = float("nan")
        raw[0] = raw[-1] = 0x7f
    qt, qx = _q(7, sum(counts), 4 * 64, "f16")
    want, got = (_run(h, c, qt, counts, 4, "f16") for c in (a, b))
    assert torch.equal(want, got)
    _compare(a, want, qx, counts, 4, "f16")


@pytest.mark.parametrize("counts", [[1, 1], [40, 3]])
def test_eight_bit_outputs(h, counts):
    c = Cache(63, "i8", 32, 2, 64, [50, 90])
    nq, rows = 4, sum(counts)
    qt, qx = _q(8, rows, nq * 64, "bf16")
    want, bar = _expect(c, qx, counts, nq, 64 ** -0.5, rows)
    g = np.random.default_rng(3)
    for kind, dt, top in (("i8", torch.int8, 127), ("f8", torch.float8_e4m3fn, 448)):
        for gran in ("fwq", "sq"):
            s = (np.abs(want).max(0 if gran == "fwq" else None) / top).reshape(-1).astype(np.float32)
            s[: s.size // 2] *= 0.9                                          # some columns saturate
            out = torch.zeros(rows, nq * 64, dtype=dt, device="cuda")
            _run(h, c, qt, counts, nq, None, out=out, gran=gran, out_scale=torch.from_numpy(s).cuda())
            y, d = want / s, bar / s * 1.01 + 1e-5
            lo, hi = BC.to_codes(y - d, kind), BC.to_codes(y + d, kind)      # rounding is monotonic
            got = out.double().cpu().numpy()
            assert np.all((got >= lo) & (got <= hi))


def test_a_scale_of_the_callers_own_and_a_bound_above_the_lengths(h):
    c = Cache(64, "i8", 64, 2, 128, [100, 5], max_len=5000)
    qt, qx = _q(9, 2, 4 * 128, "f16")
    _compare(c, _run(h, c, qt, [1, 1], 4, "f16", scale=-0.03, max_rows=100), qx, [1, 1], 4, "f16", scale=-0.03)


def test_bad_pages_rows_and_lengths_are_bounded_and_reported(h):
    c = Cache(65, "i8", 16, 1, 64, [40, 20])
    qt, qx = _q(10, 4, 64, "f16")
    c.table_t[0, 1] = 10 ** 6
    out = torch.full((4, 64), 7.0, dtype=torch.float16, device="cuda")
    ws = torch.empty(h.hero_block_attention_workspace_bytes(c.desc, 1, 4, 2), dtype=torch.uint8, device="cuda")
    h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out), 1, row_start=start_tensor([2, 2]), max_rows=2, workspace=ws)
    with pytest.raises(hero.HeroError, match="page"):
        h.check()
    c.table[0, 1] = c.n_pages - 1                                            # it is read as the nearest page
    _compare(c, out, qx, [2, 2], 1, "f16")
    c.table_t.copy_(torch.from_numpy(c.table))
    start = torch.tensor([0, 2, 9], dtype=torch.int32, device="cuda")
    h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out), 1, row_start=start, max_rows=2, workspace=ws)
    with pytest.raises(hero.HeroError, match="row range"):
        h.check()
    _compare(c, out, qx, [2, 2], 1, "f16")
    c.lens_t.copy_(torch.tensor([10 ** 6, -5], dtype=torch.int32))           # cut to max_len = 40, to 0
    out = _run(h, c, qt, [2, 2], 1, "f16")
    c.lens = [40, 0]
    _compare(c, out, qx, [2, 2], 1, "f16")


def test_a_workspace_that_is_too_small_or_missing_is_refused(h):
    c = Cache(66, "i8", 64, 1, 128, [30000])
    qt, _ = _q(11, 1, 8 * 128, "bf16")
    out = torch.empty(1, 8 * 128, dtype=torch.bfloat16, device="cuda")
    n = h.hero_block_attention_workspace_bytes(c.desc, 8, 1, 1)
    if n == 0:
        pytest.skip("this shape needs no workspace")
    for ws in (None, torch.empty(n - 16, dtype=torch.uint8, device="cuda"), torch.empty(n + 16, dtype=torch.uint8, device="cuda")[8:]):
        with pytest.raises(hero.HeroError) as e:
            h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out), 8, workspace=ws)
        assert e.value.status in (hero.ERR_WORKSPACE, hero.ERR_ALIGNMENT)


def test_a_step_as_it_is_used_eager_and_captured(h):
    """Rotation, append and attention of decode steps, chained on one stream: against the oracle on the codes the device wrote, and
    bit for bit against the same steps replayed from a CUDA graph on another stream."""
    B, nq, nkv, dh, page, steps = 3, 8, 2, 64, 16, 20
    g = np.random.default_rng(12)
    th = np.arange(64)[:, None] * 10000.0 ** (-np.arange(dh // 2) / (dh // 2))
    cos, sin = (torch.from_numpy(f(th).astype(np.float32)).cuda() for f in (np.cos, np.sin))
    gamma = torch.ones(dh, device="cuda")
    w = (nq + 2 * nkv) * dh
    inputs = [to_fp(g.standard_normal((B, w)), "bf16") for _ in range(steps)]

    def state():
        c = Cache(70, "i8", page, nkv, dh, [1, 9, 30], max_len=64)
        buf = torch.zeros(B, w, dtype=torch.bfloat16, device="cuda")
        out = torch.zeros(B, nq * dh, dtype=torch.bfloat16, device="cuda")
        pos = c.lens_t - 1
        ws = torch.empty(h.hero_block_attention_workspace_bytes(c.desc, nq, B, 1) + 1, dtype=torch.uint8, device="cuda")
        q, k, v = (hero.tensor(t) for t in (buf[:, :nq * dh], buf[:, nq * dh:(nq + nkv) * dh], buf[:, (nq + nkv) * dh:]))
        o = hero.tensor(out)

        def step():
            h.hero_qk_norm_rope(q, k, q, k, nq, nkv, pos, cos, sin, gamma, gamma)
            h.hero_block_cache_append(c.desc, k, v)
            h.hero_block_attention(c.desc, q, o, nq, workspace=ws)
        return c, buf, out, pos, step

    c, buf, out, pos, step = state()
    got, ws_keys = [], []
    for t, x in inputs:
        buf.copy_(t)
        step()
        got.append(out.clone())
        qx = buf[:, :nq * dh].double().cpu().numpy()
        for name in "kv":
            c.codes[name], c.scale[name] = c.device_codes(name), c.scale_t[name].cpu().numpy()
        c.lens = c.lens_t.cpu().tolist()
        _compare(c, out, qx, [1] * B, nq, "bf16")
        c.lens_t += 1
        pos += 1
    h.check()

    c, buf, out, pos, step = state()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
            c.lens_t += 1
            pos += 1
        for i, (t, _) in enumerate(inputs):
            buf.copy_(t)
            graph.replay()
            assert torch.equal(out, got[i]), i
    side.synchronize()
    h.check()


def test_results_do_not_depend_on_the_run(h):
    c = Cache(71, "i8", 64, 2, 128, [3000, 700, 2900], max_len=6000)
    qt, _ = _q(13, 3, 8 * 128, "bf16")
    first = _run(h, c, qt, [1] * 3, 8, "bf16")
    for _ in range(5):
        assert torch.equal(first, _run(h, c, qt, [1] * 3, 8, "bf16"))
