"""GPU: the mixture of experts where offsets pass 32 bits: weights, operands and outputs of several gigabytes, compared at sampled rows."""
import pytest
import torch

from paper_2310_17723_b200 import hero

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()
    torch.cuda.empty_cache()


def codes(*s):
    return torch.randint(-100, 101, s, dtype=torch.int8, device="cuda")


def near(got, want):
    # FP16 outputs of exact sums times FP32 factors: half a step of FP16 and a few of FP32
    return bool((got.double() - want).abs().le(want.abs() * (2.0 ** -11 + 2.0 ** -21) + 2.0 ** -25).all())


@pytest.mark.parametrize("rows", [4, 60])
def test_far_weights(h, rows):
    # 512 experts of 4096 x 1088: 2.28e9 elements; the rows of the first and the last experts
    E, N, K = 512, 4096, 1088
    w, cs = codes(E, N, K), torch.rand(E, N, device="cuda") * 1e-4
    counts = torch.zeros(E, dtype=torch.int64)
    counts[[0, 1, 493, 511]] = rows
    offset = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32).cuda()
    for pad in (0, 600 * E):                               # (capacity chooses between the two kernels)
        R = 4 * rows + pad
        a, out = codes(50, K), torch.zeros(R, N, dtype=torch.float16, device="cuda")
        token = torch.randint(0, 50, (R,), dtype=torch.int32, device="cuda")
        h.hero_moe_linear(hero.tensor(a), w, hero.tensor(out), offset, token=token, w_scale=cs)
        h.check()
        for i, e in enumerate((0, 1, 493, 511)):
            r = slice(i * rows, (i + 1) * rows)
            want = a[token[r].long()].double() @ w[e].double().T * cs[e].double()
            assert near(out[r], want)
        assert not bool(out[4 * rows:4 * rows + 1000].any())
        del out


def test_far_rows(h):
    # 1.2 million rows: A 2.5e9 bytes, out 2.4e9 elements
    R, N, K, E = 1200000, 2048, 2064, 3
    a, w, cs = torch.empty(R, K, dtype=torch.int8, device="cuda"), codes(E, N, K), torch.rand(E, N, device="cuda") * 1e-4
    for i in range(0, R, 100000):
        a[i:i + 100000] = codes(100000, K)
    offset = torch.tensor([0, 500001, 1199000, R], dtype=torch.int32, device="cuda")
    token = (R - 1 - torch.arange(R, device="cuda")).to(torch.int32)
    for gather in (True, False):
        out = torch.zeros(R, N, dtype=torch.float16, device="cuda")
        h.hero_moe_linear(hero.tensor(a), w, hero.tensor(out), offset, token=token if gather else None, w_scale=cs)
        h.check()
        for lo, e in ((0, 0), (500001, 1), (1198990, 1), (1199000, 2), (R - 8, 2)):
            rows = torch.arange(lo, lo + 8, device="cuda")
            x = a[token[rows].long() if gather else rows]
            assert near(out[rows], x.double() @ w[e].double().T * cs[e].double())
        del out


def test_far_sums(h):
    # 2.5e9 codes behind 150000 tokens
    T, k, H = 150000, 8, 2080
    R = T * k
    y = torch.empty(R, H, dtype=torch.int8, device="cuda")
    for i in range(0, R, 100000):
        y[i:i + 100000] = codes(100000, H)
    E = 4
    scale = torch.rand(E, H, device="cuda") * 0.02 + 0.01
    row = torch.randperm(R, device="cuda").to(torch.int32).reshape(T, k)
    expert = torch.randint(0, E, (T, k), dtype=torch.int32, device="cuda")
    weight = torch.rand(T, k, device="cuda")
    fp = torch.zeros(T, H, dtype=torch.float16, device="cuda")
    h.hero_moe_combine(hero.tensor(y, "fwq", scale), row, weight, expert=expert, fp_out=hero.tensor(fp))
    h.check()
    t = torch.tensor([0, 1, 777, 75000, T - 2, T - 1], device="cuda")
    v = y[row[t].long()].double() * scale.double()[expert[t].long()] * weight[t].double()[..., None]
    want, size = v.sum(1), v.abs().sum(1)
    assert bool(((fp[t].double() - want).abs() <= want.abs() * 2.0 ** -11 + size * (k + 6) * 2.0 ** -24 + 2.0 ** -25).all())
