"""GPU: the workspace that hero_block_attention_workspace_bytes asks for serves every smaller row bound."""
import pytest
import torch

from paper_2310_17723_b200 import hero
from block_util import Cache, start_tensor
from test_gpu_block_attention import _compare, _q

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


@pytest.mark.parametrize("B,nkv,group,max_len", [(4, 2, 4, 6000), (1, 1, 8, 20000), (3, 4, 1, 700), (40, 2, 8, 3000)])
def test_a_workspace_serves_every_smaller_row_bound(h, B, nkv, group, max_len):
    c = Cache(8, "i8", 64, nkv, 64, [50] * B, max_len=max_len)
    nq = nkv * group
    need = [h.hero_block_attention_workspace_bytes(c.desc, nq, 0, m) for m in range(1, 1200)]
    assert need == sorted(need)
    ws = torch.full((need[-1],), 0xff, dtype=torch.uint8, device="cuda")
    for most in (1, 3, 20, 70):
        counts = [most] + [1] * (B - 1)
        qt, qx = _q(9, sum(counts), nq * 64, "bf16")
        out = torch.full((qt.shape[0], nq * 64), 7.0, dtype=torch.bfloat16, device="cuda")
        h.hero_block_attention(c.desc, hero.tensor(qt), hero.tensor(out), nq, row_start=start_tensor(counts), max_rows=most, workspace=ws)
        h.check()
        _compare(c, out, qx, counts, nq, "bf16")
