"""Builds block caches for the GPU tests: oracle-side arrays and the device tensors that hold the same."""
import numpy as np
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import hero

Q8 = {"i8": torch.int8, "f8": torch.float8_e4m3fn}
FP = {"f16": torch.float16, "bf16": torch.bfloat16}


def to_fp(a, fp):
    """float64 array -> (device tensor of the type, float64 array of what it holds)."""
    t = torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(FP[fp])
    return t.cuda(), t.double().numpy()


class Cache:
    """kind 'i8' / 'f8'; lens per sequence; pages in shuffled order, one spare page at each end of the pool; layout 'hnd'
    ([pages, heads, page, dh]), 'nhd' ([pages, page, heads, dh]) or 'padded' (hnd with wider strides)."""

    def __init__(self, seed, kind, page, nkv, dh, lens, max_len=None, layout="hnd", spread=40.0, k_unit=None):
        g = np.random.default_rng(seed)
        self.kind, self.page, self.nkv, self.dh, self.lens = kind, page, nkv, dh, list(lens)
        B = len(lens)
        self.max_len = max_len or max(1, max(lens))
        per = -(-self.max_len // page)
        self.n_pages = n = B * per + 2
        self.table = (1 + g.permutation(B * per)).reshape(B, per).astype(np.int32)
        c = {x: BC.to_codes(g.standard_normal((n, nkv, page, dh)) * spread, kind) for x in "kv"}
        self.codes = c
        k_unit = k_unit if k_unit is not None else 1.5 / spread
        self.scale = {"k": (k_unit * np.exp(0.5 * g.standard_normal((n, nkv)))).astype(np.float32),
                      "v": (1 / spread * np.exp(0.5 * g.standard_normal((n, nkv)))).astype(np.float32)}
        self.buf = {x: self._device(c[x], layout) for x in "kv"}
        self.scale_t = {x: torch.from_numpy(self.scale[x].copy()).cuda() for x in "kv"}
        self.table_t = torch.from_numpy(self.table).cuda()
        self.lens_t = torch.tensor(self.lens, dtype=torch.int32, device="cuda")
        self.desc = hero.block_cache(self.buf["k"], self.buf["v"], self.scale_t["k"], self.scale_t["v"], self.table_t, self.lens_t, self.max_len)

    def _device(self, codes, layout):
        t = torch.from_numpy(codes.astype(np.float32)).to(Q8[self.kind]).cuda()
        if layout == "nhd":
            return t.view(torch.uint8).transpose(1, 2).contiguous().view(Q8[self.kind]).transpose(1, 2)
        if layout == "padded":
            n, h, p, d = t.shape
            wide = torch.zeros(n, h + 1, p + 3, d + 16, dtype=torch.uint8, device="cuda").view(Q8[self.kind])
            v = wide[:, :h, :p, :d]
            v.view(torch.uint8).copy_(t.view(torch.uint8))
            return v
        return t

    def set_lens(self, lens):
        self.lens = list(lens)
        self.lens_t.copy_(torch.tensor(self.lens, dtype=torch.int32))

    def device_codes(self, x):
        return self.buf[x].float().cpu().numpy().astype(np.float64)

    def values(self, x, b):
        """[len, heads, dh] of sequence b."""
        return BC.tokens(self.codes[x], self.scale[x], self.table[b], max(self.lens[b], 0), self.page)


def starts(counts):
    return [0] + list(np.cumsum(counts))


def start_tensor(counts):
    return torch.tensor(starts(counts), dtype=torch.int32, device="cuda")
