"""Refusals of the Python binding that are made before anything reaches the library (no GPU)."""
import pytest
import torch

from paper_2310_17723_b200 import hero


def on_nowhere(t, gran="none", scale=None):
    """What hero.tensor gives, of a CPU tensor: device -1, as torch numbers it."""
    T = hero.Tensor(t.data_ptr(), hero._DT[t.dtype], hero.GRAN[gran], t.shape[0], t.shape[1], t.stride(0), None if scale is None else scale.data_ptr())
    T._keep, T._device = (t, scale), -1
    return T


class Library:
    """Takes every call and does nothing."""

    def __getattr__(self, name):
        return lambda *a: self.calls.append(name) or hero.OK

    def __init__(self):
        self.calls = []


@pytest.fixture
def h(monkeypatch):
    hd = hero.Handle.__new__(hero.Handle)
    hd._h, hd._device, hd._lib = None, -1, Library()
    monkeypatch.setattr(hd, "_raw_stream", lambda s: 0, raising=False)
    return hd


@pytest.mark.parametrize("gather", [False, True])
@pytest.mark.parametrize("rows,entries,refused", [(8, 7, True), (8, 0, True), (8, 8, False), (8, 9, False)])
def test_a_token_wise_scale_reaches_the_last_row_of_the_grouped_products(h, gather, rows, entries, refused):
    A, out = torch.zeros(rows, 64, dtype=torch.int8), torch.zeros(8, 96, dtype=torch.float16)
    W, offset, token = torch.zeros(3, 96, 64, dtype=torch.int8), torch.zeros(4, dtype=torch.int32), torch.zeros(8, dtype=torch.int32)
    call = lambda: h.hero_moe_linear(on_nowhere(A, "twq", torch.ones(entries)), W, on_nowhere(out), offset, token=token if gather else None, w_scale=torch.ones(3, 96))  # noqa: E731
    if refused:
        with pytest.raises(hero.HeroError, match="scale"):
            call()
    else:
        call()
    assert h._lib.calls == ([] if refused else ["hero_moe_linear"])


@pytest.mark.parametrize("entries,refused", [(7, True), (8, False), (9, False)])
def test_a_token_wise_scale_reaches_the_last_row_of_the_dense_products(h, monkeypatch, entries, refused):
    monkeypatch.setattr(hero, "lib", lambda: h._lib)
    monkeypatch.setattr(hero, "_stream", lambda s: None)
    A, out, W = torch.zeros(8, 64, dtype=torch.int8), torch.zeros(8, 96, dtype=torch.float16), torch.zeros(96, 64, dtype=torch.int8)
    call = lambda: h.hero_w8a8_linear(on_nowhere(A, "twq", torch.ones(entries)), W, on_nowhere(out), w_scale=torch.ones(96))  # noqa: E731
    if refused:
        with pytest.raises(hero.HeroError, match="scale"):
            call()
    else:
        call()
    assert h._lib.calls == ([] if refused else ["hero_w8a8_linear"])
