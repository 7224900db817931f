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
