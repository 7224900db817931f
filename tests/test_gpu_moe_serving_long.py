"""GPU: the expert part of a layer as test_gpu_moe_serving runs it, with as many tokens as take the router's two kernels, the products of CTA pairs and the combine's ring."""
import pytest
import torch

from paper_2310_17723_b200 import hero
import test_gpu_moe_serving as serving

pytestmark = pytest.mark.gpu
MOST = 900                                                # 2700 rows for 16 experts (pairs above 32 a piece), above four tokens for each of 148 SMs


@pytest.fixture(scope="module")
def h():
    hd = hero.Handle()
    yield hd
    hd.check()
    hd.close()


@pytest.mark.parametrize("kind", ["i8", "f8"])
def test_a_long_batch_eager_and_replayed(h, kind, monkeypatch):
    monkeypatch.setattr(serving, "MOST", MOST)
    b = serving.Block(h, 11, kind)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            b.call()
    for run, seed, n in ((b.call, 1, MOST), (graph.replay, 2, MOST), (graph.replay, 3, 611), (graph.replay, 4, 1), (graph.replay, 5, 0), (b.call, 6, 899)):
        b.feed(seed, n)
        run()
        h.check()
        b.check(n)


def test_two_long_batches_on_two_streams_at_once(h, monkeypatch):
    monkeypatch.setattr(serving, "MOST", MOST)
    blocks, streams = [serving.Block(h, s, "i8") for s in (12, 13)], [torch.cuda.Stream() for _ in range(2)]
    for i, b in enumerate(blocks):
        b.feed(40 + i, MOST - 200 * i)
    torch.cuda.synchronize()
    for _ in range(20):
        for b, s in zip(blocks, streams):
            with torch.cuda.stream(s):
                b.call()
    torch.cuda.synchronize()
    h.check()
    for i, b in enumerate(blocks):
        b.check(MOST - 200 * i)
