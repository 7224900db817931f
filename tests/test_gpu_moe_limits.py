"""GPU: the mixture of experts at the most rows and tokens that 32 bits can number."""
import pytest
import torch

from paper_2310_17723_b200 import hero

pytestmark = pytest.mark.gpu
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def h():
    torch.cuda.empty_cache()
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()
    torch.cuda.empty_cache()


def test_one_expert_with_the_most_rows(h):
    # 2^31 - 1 rows of 16 features, out 34 GB: row r has A's row r mod 251, so that each output row is one of 251
    N = K = 16
    a = torch.randint(-100, 101, (251, K), dtype=torch.int8, device="cuda")
    w = torch.randint(-100, 101, (1, N, K), dtype=torch.int8, device="cuda")
    token = torch.arange(MOST, dtype=torch.int32, device="cuda").remainder_(251)
    out = torch.zeros(MOST, N, dtype=torch.int8, device="cuda")
    cs = torch.full((1, N), 1.0 / 1024, device="cuda")     # (a power of two: the products are exact)
    h.hero_moe_linear(hero.tensor(a), w, hero.tensor(out), torch.tensor([0, MOST], dtype=torch.int32, device="cuda"), token=token, w_scale=cs)
    h.check()
    want = (a.double() @ w[0].double().T / 1024).round().clamp(-127, 127).to(torch.int8)         # (ties to even)
    step = 251 * (1 << 20)
    for lo in range(0, MOST, step):
        got = out[lo:lo + step]
        full = got.shape[0] // 251 * 251
        assert bool((got[:full].view(-1, 251, N) == want).all()), lo
        assert torch.equal(got[full:], want[:got.shape[0] - full])


def plan(x, k):
    """Top k of the rows of x in torch: experts, offsets, tokens of the sorted rows, row of each pair."""
    T, E = x.shape
    e = torch.sort(x.double(), dim=-1, descending=True, stable=True)[1][:, :k]
    by, at = torch.sort(e.reshape(-1), stable=True)
    row = torch.empty_like(at)
    row[at] = torch.arange(T * k, device="cuda")
    return e.int(), torch.searchsorted(by, torch.arange(E + 1, device="cuda")).int(), (at // k).int(), row.reshape(T, k).int()


@pytest.mark.parametrize("T,E,k,n", [(151552, 8, 2, None), (151553, 8, 2, None), (160001, 300, 3, None), (303105, 40, 8, 200000), (1500000, 17, 1, None)])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_more_tokens_than_the_sms_have_chunks_for(h, T, E, k, n, dt):
    # (above 1024 tokens for each of 148 SMs a third kernel adds the counts up)
    x = torch.randn(T, E, device="cuda", generator=torch.Generator("cuda").manual_seed(T)).to(dt)
    i32 = dict(dtype=torch.int32, device="cuda")
    expert, row, weight = torch.full((T, k), 7, **i32), torch.full((T, k), 7, **i32), torch.full((T, k), 7.0, device="cuda")
    offset, token = torch.full((E + 1,), 7, **i32), torch.full((T * k,), 7, **i32)
    bytes_ = h.hero_moe_route_workspace_bytes(T, E, k)
    ws = torch.full((bytes_ + 256,), 0xaa, dtype=torch.uint8, device="cuda")
    for _ in range(2):                                     # (the second call finds what the first one left)
        h.hero_moe_route(hero.tensor(x), expert, weight, offset, token, row, renorm=True, n_tokens=None if n is None else torch.tensor([n], **i32), workspace=ws[:bytes_])
        h.check()
        N = T if n is None else n
        e, o, t, r = plan(x[:N], k)
        assert torch.equal(expert[:N], e) and torch.equal(offset, o) and torch.equal(token[:N * k], t) and torch.equal(row[:N], r)
        w = torch.softmax(x[:N].double().gather(1, e.long()), -1)
        assert bool(((weight[:N] - w).abs() <= 4e-6 * w).all())              # (two exponentials, a sum of up to 8 and a quotient: below 64 units of 2^-24)
        assert bool((expert[N:] == -1).all()) and bool((row[N:] == -1).all()) and bool((weight[N:] == 0).all()) and bool((token[N * k:] == 7).all())
        assert bool((ws[bytes_:] == 0xaa).all())


def test_the_most_tokens(h):
    # 2^31 - 1 tokens of one expert: every row is its token
    T = MOST
    assert h.hero_moe_route_workspace_bytes(T, 1, 1) < 1 << 24
    x = torch.zeros(T, 1, dtype=torch.bfloat16, device="cuda")
    i32 = dict(dtype=torch.int32, device="cuda")
    expert, row, token = (torch.full(s, 7, **i32) for s in ((T, 1), (T, 1), (T,)))
    weight, offset = torch.zeros(T, 1, device="cuda"), torch.zeros(2, **i32)
    ws = torch.empty(h.hero_moe_route_workspace_bytes(T, 1, 1), dtype=torch.uint8, device="cuda")
    h.hero_moe_route(hero.tensor(x), expert, weight, offset, token, row, workspace=ws)
    h.check()
    assert offset.tolist() == [0, T]
    step = 1 << 28
    for lo in range(0, T, step):
        want = torch.arange(lo, min(lo + step, T), **i32)
        r = slice(lo, lo + want.numel())
        assert torch.equal(token[r], want) and torch.equal(row[r, 0], want) and bool((expert[r] == 0).all()) and bool((weight[r] == 1).all())
