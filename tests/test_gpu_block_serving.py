"""GPU: the operators of the block cache as a server runs them, between two 8-bit linears and without a wait on the host: projection of queries,
keys and values (hero_w8a8_linear, 16-bit out), norm and rotation, append, attention with an 8-bit output, output projection
(hero_w8a8_linear).  A prompt, a few drafted tokens, then single tokens, all from one workspace; every stage is compared with the
oracle on what the stage before it left on the device, within that stage's own bounds."""
import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from oracle import ops as O
from paper_2310_17723_b200 import hero
from block_util import Cache, Q8, start_tensor, starts
from test_gpu_block_attention import _expect
from test_gpu_qk_rope import _bound, _tables

pytestmark = pytest.mark.gpu

HIDDEN, NQ, NKV, DH, PAGE, MAX_LEN = 256, 4, 2, 64, 16, 700
STEPS = [[40, 5, 17], [3, 1, 1]] + [[1, 1, 1]] * 6 + [[0, 30, 2], [1, 0, 1]]


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


def _codes(g, kind, *shape):
    """8-bit codes, as a device tensor and as the numbers they stand for."""
    x = BC.to_codes(g.standard_normal(shape) * (40.0 if kind == "i8" else 60.0), kind)
    return torch.from_numpy(x.astype(np.float32)).to(Q8[kind]).cuda(), (x.astype(np.int8) if kind == "i8" else x)


def _gemm(kind, x, w, scale, rows=None):
    f = O.gemm_quant if kind == "i8" else O.gemm_quant_f8
    return f(O.QT(kind, x, row_scale=rows), w.T, scale, None, "none", O.OutSpec("fp", dtype="f32")).data


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_server_between_two_linears(h, kind, graph):
    g = np.random.default_rng(1)
    width, B = (NQ + 2 * NKV) * DH, 3
    w1t, w1 = _codes(g, kind, width, HIDDEN)
    w2t, w2 = _codes(g, kind, HIDDEN, NQ * DH)
    s1, s2 = (g.uniform(0.5, 1.5, n).astype(np.float32) * 1e-3 for n in (width, HIDDEN))
    s1t, s2t = torch.from_numpy(s1).cuda(), torch.from_numpy(s2).cuda()
    o_scale = np.full(NQ * DH, 0.02 if kind == "i8" else 0.005, np.float32) * g.uniform(0.5, 2.0, NQ * DH).astype(np.float32)
    o_scale_t = torch.from_numpy(o_scale).cuda()
    cos, sin, cos_t, sin_t = _tables(MAX_LEN, DH)
    gamma = (1 + 0.2 * g.standard_normal(DH)).astype(np.float32)
    gamma_t = torch.from_numpy(gamma).cuda()
    c = Cache(2, kind, PAGE, NKV, DH, [0] * B, max_len=MAX_LEN)
    codes, scale = ({x: getattr(c, n)[x].copy() for x in "kv"} for n in ("codes", "scale"))
    most = max(max(n) for n in STEPS)
    ws = torch.full((h.hero_block_attention_workspace_bytes(c.desc, NQ, 0, most),), 0xff, dtype=torch.uint8, device="cuda")
    # every step's buffers, before the first call
    steps, lens = [], np.zeros(B, int)
    for n in STEPS:
        rows, lens = sum(n), lens + n
        xt, x = _codes(g, kind, rows, HIDDEN)
        r = (g.uniform(0.5, 2.0, rows) * 0.02).astype(np.float32)
        pos = np.concatenate([np.arange(a - m, a) for a, m in zip(lens, n)]).astype(np.int32)
        new = lambda cols, dt: torch.zeros(rows, cols, dtype=dt, device="cuda")  # noqa: E731
        steps.append(dict(n=n, lens=list(lens), x=x, r=r, pos=pos, xt=xt, rt=torch.from_numpy(r).cuda(), post=torch.from_numpy(pos).cuda(),
                          nt=torch.tensor(n, dtype=torch.int32, device="cuda"), start=start_tensor(n), qkv=new(width, torch.float16),
                          q=new(NQ * DH, torch.float16), k=new(NKV * DH, torch.float16), a=new(NQ * DH, Q8[kind]), y=new(HIDDEN, torch.float16)))

    def call(s):
        qkv, a, b = s["qkv"], NQ * DH, (NQ + NKV) * DH
        c.lens_t.add_(s["nt"])
        h.hero_w8a8_linear(hero.tensor(s["xt"], "twq", s["rt"]), w1t, hero.tensor(qkv), w_scale=s1t)
        h.hero_qk_norm_rope(hero.tensor(qkv[:, :a]), hero.tensor(qkv[:, a:b]), hero.tensor(s["q"]), hero.tensor(s["k"]), NQ, NKV, s["post"], cos_t, sin_t,
                            gamma_t, gamma_t, 1e-5, "adjacent")
        h.hero_block_cache_append(c.desc, hero.tensor(s["k"]), hero.tensor(qkv[:, b:]), row_start=s["start"], max_rows=max(s["n"]))
        h.hero_block_attention(c.desc, hero.tensor(s["q"]), hero.tensor(s["a"], "fwq", o_scale_t), NQ, row_start=s["start"], max_rows=max(s["n"]), workspace=ws)
        h.hero_w8a8_linear(hero.tensor(s["a"]), w2t, hero.tensor(s["y"]), w_scale=s2t)

    if graph:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured, stream=side):
                for s in steps:
                    call(s)
            for x in "kv":                                                   # (nothing ran during the capture)
                assert torch.equal(c.scale_t[x].cpu(), torch.from_numpy(scale[x]))
            captured.replay()
    else:
        for s in steps:
            call(s)
    torch.cuda.synchronize()
    h.check()

    num = lambda t: t.float().cpu().numpy().astype(np.float64)  # noqa: E731
    half = 2.0 ** -11                                                        # half a step of FP16
    for s in steps:
        qkv, q, k, a, y = (num(s[x]) for x in ("qkv", "q", "k", "a", "y"))
        want = _gemm(kind, s["x"], w1, s1, s["r"])
        size = np.abs(np.asarray(s["x"], np.float64)) @ np.abs(np.asarray(w1, np.float64)).T * s["r"][:, None] * s1
        # INT8 sums are exact; e4m3 products are, their FP32 sums are not
        assert np.all(np.abs(qkv - want) <= half * np.abs(want) + (8 if kind == "i8" else HIDDEN + 8) * 2.0 ** -24 * size + 2.0 ** -25)
        at, to = NQ * DH, (NQ + NKV) * DH
        for got, x, heads in ((q, qkv[:, :at], NQ), (k, qkv[:, at:to], NKV)):
            w, bar = _bound(x, heads, gamma, 1e-5, cos, sin, s["pos"], "adjacent", "f16")
            assert np.all(np.abs(got - w) <= bar)
        for x, rows in (("k", k), ("v", qkv[:, to:])):
            codes[x], scale[x] = BC.append(codes[x], scale[x], c.table, s["lens"], s["n"], starts(s["n"]), rows, PAGE, kind)
        c.codes, c.scale, c.lens = codes, scale, s["lens"]
        w, bar = _expect(c, q, s["n"], NQ, DH ** -0.5, q.shape[0])
        v, d = w / o_scale, bar / o_scale * 1.01 + 1e-5
        assert np.all((a >= BC.to_codes(v - d, kind)) & (a <= BC.to_codes(v + d, kind)))           # rounding is monotonic
        want = _gemm(kind, a.astype(np.int8) if kind == "i8" else a, w2, s2)
        size = np.abs(a) @ np.abs(np.asarray(w2, np.float64)).T * s2
        assert np.all(np.abs(y - want) <= half * np.abs(want) + (8 if kind == "i8" else NQ * DH + 8) * 2.0 ** -24 * size + 2.0 ** -25)
    for x in "kv":
        assert np.array_equal(c.device_codes(x), codes[x]) and np.array_equal(c.scale_t[x].cpu().numpy(), scale[x])
