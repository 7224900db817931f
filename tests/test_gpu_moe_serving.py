"""GPU: a mixture of experts as a layer runs it: LN^quant, router projection (hero_w8a8_linear), route, FC1 with its gated activation, FC2, combine with the
next LN^quant, eager and as one captured graph that is replayed with other tokens, more and fewer of them; on two streams at once.  Every stage is
compared with the oracle on what the stage before it left on the device, within that stage's own bounds."""
import numpy as np
import pytest
import torch

from oracle import moe as M
from oracle import ops as O
from paper_2310_17723_b200 import hero
from moe_util import STEP, TINY, U, assert_near, f32, linear_bounds, num, to

pytestmark = pytest.mark.gpu

H, F, E, K, MOST = 256, 128, 16, 3, 140


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


class Block:
    """Weights of one layer's expert part and the buffers of a padded batch of MOST tokens."""

    def __init__(self, h, seed, kind):
        g = np.random.default_rng(seed)
        self.h, self.kind = h, kind
        size = 36 if kind == "i8" else 60
        q8 = lambda *s: to(g.standard_normal(s) * size, kind)  # noqa: E731
        self.wr, self.wr_n = q8(E, H)
        self.w1, self.w1_n = q8(E, 2 * F, H)
        self.w2, self.w2_n = q8(E, H, F)
        self.cr, self.cr_n = f32(np.exp(0.2 * g.standard_normal(E)) / (size * 16))
        self.c1, self.c1_n = f32(np.exp(0.2 * g.standard_normal((E, 2 * F))) / (size * 16))
        self.p1, self.p1_n = f32((30 if kind == "i8" else 100) * np.exp(0.2 * g.standard_normal((E, F))))
        self.c2, self.c2_n = f32(np.exp(0.2 * g.standard_normal((E, H))) / (size * size * 12))
        self.b1, self.b1_n = f32(0.1 * g.standard_normal((E, 2 * F)))
        self.b2, self.b2_n = f32(0.1 * g.standard_normal((E, H)))
        self.g1, self.g1_n = f32(1 + 0.2 * g.standard_normal(H))
        self.be, self.be_n = f32(0.1 * g.standard_normal(H))
        dt = self.wr.dtype
        new = lambda *s, d=torch.float16: torch.full(s, 3.0, device="cuda").to(d)  # noqa: E731
        i32 = lambda *s: torch.full(s, 77, dtype=torch.int32, device="cuda")  # noqa: E731
        self.h_in, self.n = new(MOST, H), torch.zeros(1, dtype=torch.int32, device="cuda")
        self.x, self.xs, self.logits = new(MOST, H, d=dt), new(MOST, d=torch.float32), new(MOST, E)
        self.expert, self.row, self.weight = i32(MOST, K), i32(MOST, K), new(MOST, K, d=torch.float32)
        self.offset, self.token = i32(E + 1), i32(MOST * K)
        self.hid, self.y = new(MOST * K, F, d=dt), new(MOST * K, H)
        self.h_out, self.x2, self.x2s = new(MOST, H), new(MOST, H, d=dt), new(MOST, d=torch.float32)
        self.ws = torch.full((h.hero_moe_route_workspace_bytes(MOST, E, K),), 0xff, dtype=torch.uint8, device="cuda")

    def call(self):
        h, t = self.h, hero.tensor
        h.hero_layernorm_quant(t(self.h_in), self.g1, self.be, 1e-5, t(self.x, "twq", self.xs))
        h.hero_w8a8_linear(t(self.x, "twq", self.xs), self.wr, t(self.logits), w_scale=self.cr)
        h.hero_moe_route(t(self.logits), self.expert, self.weight, self.offset, self.token, self.row, n_tokens=self.n, workspace=self.ws)
        h.hero_moe_linear(t(self.x, "twq", self.xs), self.w1, t(self.hid), self.offset, token=self.token, w_scale=self.c1, bias=self.b1, act="silu", gated=True,
                          post_scale=self.p1)
        h.hero_moe_linear(t(self.hid), self.w2, t(self.y), self.offset, w_scale=self.c2, bias=self.b2)
        h.hero_moe_combine(t(self.y), self.row, self.weight, residual=t(self.h_in), fp_out=t(self.h_out), out=t(self.x2, "twq", self.x2s), gamma=self.g1,
                           beta=self.be, eps=1e-5)

    def check(self, n):
        x, xs = num(self.x), num(self.xs)
        e, w, offset, token, row = M.route(num(self.logits), K, n_tokens=n)
        assert np.array_equal(self.expert.cpu().numpy(), e) and np.array_equal(self.row.cpu().numpy(), row)
        assert np.array_equal(self.offset.cpu().numpy(), offset) and np.array_equal(self.token.cpu().numpy()[:len(token)], token)
        assert np.allclose(num(self.weight), w, rtol=3e-6, atol=1e-30)
        R = len(token)
        y, v, size = M.linear(x, xs, self.w1_n, self.c1_n, self.b1_n, "silu", True, self.p1_n, offset, token)
        hid = num(self.hid)
        assert_near(hid[:R], y, linear_bounds(y, v, size, "silu", True, self.p1_n, self.kind, H, offset), self.kind)
        y, v, size = M.linear(hid, None, self.w2_n, self.c2_n, self.b2_n, "none", False, None, offset, None)
        got = num(self.y)
        assert_near(got[:R], y, linear_bounds(y, v, size, "none", False, None, self.kind, F, offset), "f16")
        r, size = M.combine(got, row, num(self.weight), residual=num(self.h_in))
        out, bar = num(self.h_out), (K + 6) * U * size
        assert np.all(np.abs(out - r) <= bar + STEP["f16"] * (np.abs(r) + bar) + TINY["f16"])
        want = O.layernorm(out, self.g1_n.astype(np.float64), self.be_n.astype(np.float64), 1e-5)
        top, s = (127 if self.kind == "i8" else 448), num(self.x2s)
        assert np.allclose(s, np.abs(want).max(1) / top, rtol=1e-5)
        q, d = want / s[:, None], 2e-5 * (np.abs(want / s[:, None]) + top / 4)             # 70 roundings of FP32 relative to the row's size
        assert np.all((num(self.x2) >= M.emit(q - d, self.kind)) & (num(self.x2) <= M.emit(q + d, self.kind)))

    def feed(self, seed, n):
        g = np.random.default_rng(seed)
        self.h_in.copy_(torch.from_numpy((2 * g.standard_normal((MOST, H))).astype(np.float32)))
        self.n.fill_(n)


@pytest.mark.parametrize("kind", ["i8", "f8"])
@pytest.mark.parametrize("graph", [False, True])
def test_the_expert_part_of_a_layer(h, kind, graph):
    b = Block(h, 1, kind)
    run = b.call
    if graph:
        side = torch.cuda.Stream()
        with torch.cuda.stream(side):
            captured = torch.cuda.CUDAGraph()
            with torch.cuda.graph(captured, stream=side):
                b.call()
        run = captured.replay
    for seed, n in ((1, MOST), (2, 1), (3, 77), (4, 0), (5, MOST)):
        b.feed(seed, n)
        run()
        h.check()
        b.check(n)


def test_two_layers_on_two_streams_at_once(h):
    blocks, streams = [Block(h, s, "i8") for s in (2, 3)], [torch.cuda.Stream() for _ in range(2)]
    for i, b in enumerate(blocks):
        b.feed(10 + i, 100 + 40 * i)
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.call()
    torch.cuda.synchronize()
    h.check()
    for i, b in enumerate(blocks):
        b.check(100 + 40 * i)


def test_two_graphs_that_share_a_workspace_one_after_the_other(h):
    # (at the same time they would need one each)
    blocks = [Block(h, s, "i8") for s in (4, 5)]
    blocks[1].ws = blocks[0].ws
    graphs = []
    for i, b in enumerate(blocks):
        b.feed(20 + i, 120)
        side, g = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.stream(side):
            with torch.cuda.graph(g, stream=side):
                b.call()
        graphs.append(g)
    for _ in range(5):
        for g in graphs:
            g.replay()
    h.check()
    for b in blocks:
        b.check(120)


def test_an_explicit_stream(h):
    b, s = Block(h, 6, "i8"), torch.cuda.Stream()
    b.feed(30, 90)
    b.call()
    h.check()
    want = [getattr(b, n).clone() for n in ("expert", "weight", "offset", "hid", "h_out")]
    for n in ("expert", "weight", "offset", "hid", "h_out"):
        getattr(b, n).zero_()
    s.wait_stream(torch.cuda.current_stream())
    t = hero.tensor
    h.hero_moe_route(t(b.logits), b.expert, b.weight, b.offset, b.token, b.row, n_tokens=b.n, workspace=b.ws, stream=s)
    h.hero_moe_linear(t(b.x, "twq", b.xs), b.w1, t(b.hid), b.offset, token=b.token, w_scale=b.c1, bias=b.b1, act="silu", gated=True, post_scale=b.p1, stream=s)
    h.hero_moe_linear(t(b.hid), b.w2, t(b.y), b.offset, w_scale=b.c2, bias=b.b2, stream=s)
    h.hero_moe_combine(t(b.y), b.row, b.weight, residual=t(b.h_in), fp_out=t(b.h_out), stream=s)
    s.synchronize()
    h.check()
    used = int(b.offset[-1])
    for n, w in zip(("expert", "weight", "offset", "hid", "h_out"), want):
        got = getattr(b, n)
        assert torch.equal(got[:used], w[:used]) if n == "hid" else torch.equal(got, w)


def test_tensors_of_another_device_are_refused(h):
    b = Block(h, 7, "i8")
    t, own = hero.tensor, h._device
    x, y, out = t(b.x, "twq", b.xs), t(b.y), t(b.h_out)
    h._device = own + 1
    try:
        for f in (lambda: h.hero_moe_route(t(b.logits), b.expert, b.weight, b.offset, b.token, b.row, workspace=b.ws),
                  lambda: h.hero_moe_linear(x, b.w1, t(b.hid), b.offset, token=b.token, w_scale=b.c1, gated=True),
                  lambda: h.hero_moe_combine(y, b.row, b.weight, fp_out=out)):
            with pytest.raises(hero.HeroError, match="device"):
                f()
    finally:
        h._device = own
