"""The oracle of the block cache pinned to library float64 routines and to the definition's own consequences; the entry
points' refusals, which need no GPU because they come before anything is launched."""
import ctypes as C

import numpy as np
import pytest
import torch

from oracle import block_cache as BC
from paper_2310_17723_b200 import build as B
from paper_2310_17723_b200 import hero


def test_append_keeps_every_value_within_half_a_step_and_grows_scales_only():
    g = np.random.default_rng(1)
    pages, heads, page, dh = 5, 2, 16, 64
    codes, scale = np.zeros((pages, heads, page, dh)), np.full((pages, heads), 9.0, np.float32)
    table, x = [[3, 1, 0]], g.standard_normal((40, heads * dh)).astype(np.float32)
    for kind in ("i8", "f8"):
        c, s = codes, scale
        at = 0
        for n in (1, 4, 20, 15):                       # 40 tokens in four calls, over page borders
            c, s2 = BC.append(c, s, table, [at + n], [n], [0], x[at:at + n], page, kind)
            assert at == 0 or np.all(s2[[3, 1, 0]] >= 0)
            s = s2
            at += n
        y = BC.tokens(c, s, table[0], 40, page).reshape(40, -1)
        # each requantisation is off by half a step of the scale then in force (e4m3: half of 2^-3 relative at most), and a
        # page of these three saw at most three
        step = np.repeat(BC.tokens(np.ones_like(c), s, table[0], 40, page).reshape(40, -1), 1, axis=1)
        bar = 3 * (0.5 * step if kind == "i8" else 0.5 * 0.125 * np.abs(x) + step * 2.0 ** -10)
        assert np.all(np.abs(y - x) <= bar * 1.01)
        assert np.all(s[[2, 4]] == 9.0) and np.all(c[[2, 4]] == 0)          # pages of nobody are untouched


def test_append_edge_values():
    page, dh = 16, 64
    x = np.zeros((2, dh), np.float32)
    c, s = BC.append(np.ones((1, 1, page, dh)), np.ones((1, 1)), [[0]], [2], [2], [0], x, page, "i8")
    assert s[0, 0] == 0 and np.all(c[0, 0, :2] == 0) and np.all(c[0, 0, 2:] == 1)
    x[0, 0], x[0, 1], x[1, 2], x[1, 3] = np.nan, np.inf, -np.inf, 3.0
    c, s = BC.append(np.ones((1, 1, page, dh)), np.ones((1, 1)), [[0]], [2], [2], [0], x, page, "i8")
    assert s[0, 0] == np.float32(3.0) / np.float32(127) and list(c[0, 0, 0, :2]) == [0, 127] and list(c[0, 0, 1, 2:4]) == [-127, 127]


def test_attention_against_the_library_routine():
    g = np.random.default_rng(2)
    n, L, nq, nkv, dh = 3, 11, 4, 2, 8
    q, k, v = g.standard_normal((n, nq, dh)), g.standard_normal((L, nkv, dh)), g.standard_normal((L, nkv, dh))
    o, _, _ = BC.attention(q, k, v, nq // nkv, 0.3)
    t = [torch.from_numpy(np.ascontiguousarray(a.transpose(1, 0, 2))) for a in (q, np.repeat(k, 2, 1), np.repeat(v, 2, 1))]
    mask = torch.ones(n, L, dtype=torch.bool).tril(L - n)
    want = torch.nn.functional.scaled_dot_product_attention(*t, attn_mask=mask, scale=0.3).numpy().transpose(1, 0, 2)
    assert np.allclose(o, want, rtol=1e-12, atol=1e-12)
    o, _, _ = BC.attention(q, k[:2], v[:2], 2, 0.3)                          # the first row has no token: zeros
    assert np.all(o[0] == 0) and np.all(o[1] != 0)


@pytest.mark.parametrize("pairing", ["halves", "adjacent"])
def test_rotation_is_a_complex_product_and_keeps_norms(pairing):
    g = np.random.default_rng(3)
    rows, heads, dh, rot = 5, 3, 32, 16
    x, th = g.standard_normal((rows, heads * dh)), g.uniform(0, 7, (9, rot // 2))
    pos = np.array([0, 8, 3, 3, 1])
    y = BC.norm_rope(x, heads, None, 0.0, np.cos(th), np.sin(th), pos, pairing).reshape(rows, heads, dh)
    x = x.reshape(rows, heads, dh)
    a = x[..., :8] + 1j * x[..., 8:16] if pairing == "halves" else x[..., 0:16:2] + 1j * x[..., 1:16:2]
    z = a * np.exp(1j * th[pos])[:, None]
    got = y[..., :8] + 1j * y[..., 8:16] if pairing == "halves" else y[..., 0:16:2] + 1j * y[..., 1:16:2]
    assert np.allclose(got, z) and np.array_equal(y[..., rot:], x[..., rot:])


# ---------------------------------------------------------------------------------------------------- refusals
@pytest.fixture(scope="module")
def call():
    """Calls an entry point with a blank handle: every refusal is made before the handle's device is looked at."""
    B.build()
    blank = (C.c_uint8 * (1 << 20))()
    def run(name, *structs):
        status = getattr(hero.lib(), name)(C.cast(blank, C.c_void_p), *[C.byref(s) for s in structs], None)
        return status, hero.lib().hero_last_error().decode()
    return run


P = 1 << 20                      # a 16-byte aligned address that nothing looks at


def _cache(**kw):
    d = dict(k=P, v=P, k_scale=P, v_scale=P, dtype=hero.I8, page=64, n_pages=10, page_stride=2 * 64 * 128, head_stride=64 * 128, ld=128,
             table=P, ld_table=4, len=P, max_len=256, B=2, nkv=2, dh=128)
    d.update(kw)
    return hero.BlockCache(**d)


def _t(rows, cols, dtype=hero.BF16, gran=0, scale=None, data=P, ld=None):
    return hero.Tensor(data, dtype, gran, rows, cols, cols if ld is None else ld, scale)


BAD_CACHE = [dict(page=48), dict(dh=96), dict(dtype=hero.F16), dict(nkv=0), dict(max_len=0), dict(max_len=257), dict(n_pages=0), dict(k=None),
             dict(v_scale=None), dict(table=None), dict(len=None), dict(k=P + 8), dict(ld=136), dict(ld=112), dict(head_stride=8), dict(page_stride=24),
             dict(B=-1), dict(B=70000), dict(n_pages=1 << 31)]


@pytest.mark.parametrize("bad", BAD_CACHE)
def test_a_bad_cache_is_refused_by_every_entry_point(call, bad):
    c = _cache(**bad)
    nkv = max(c.nkv, 1)
    rows = hero.BlockRowsArgs(_t(4, nkv * c.dh), _t(4, nkv * c.dh), P, 2)
    for name in ("hero_block_cache_append", "hero_block_cache_read"):
        assert call(name, c, rows)[0] not in (hero.OK, hero.ERR_CUDA), name
    a = hero.BlockAttnArgs(_t(4, 4 * c.dh), _t(4, 4 * c.dh), P, 2, 4, 0.0, P, 1 << 30)
    assert call("hero_block_attention", c, a)[0] not in (hero.OK, hero.ERR_CUDA)


@pytest.mark.parametrize("k,v,start,most", [
    (_t(4, 255), _t(4, 256), P, 2), (_t(4, 256), _t(5, 256), P, 2), (_t(4, 256, hero.F16), _t(4, 256), P, 2),
    (_t(4, 256, hero.F32), _t(4, 256, hero.F32), P, 2), (_t(4, 256), _t(4, 256), P, 0), (_t(4, 256), _t(4, 256), None, 2),
    (_t(1, 256), _t(1, 256), None, 1), (_t(4, 256, data=P + 2), _t(4, 256), P, 2), (_t(4, 256, ld=257), _t(4, 256), P, 2)])
def test_bad_rows_are_refused(call, k, v, start, most):
    for name in ("hero_block_cache_append", "hero_block_cache_read"):
        assert call(name, _cache(), hero.BlockRowsArgs(k, v, start, most))[0] not in (hero.OK, hero.ERR_CUDA), name


def test_nothing_to_do_is_no_error(call):
    empty = _t(0, 256, data=None)
    assert call("hero_block_cache_append", _cache(), hero.BlockRowsArgs(empty, empty, P, 2))[0] == hero.OK
    assert call("hero_block_cache_read", _cache(), hero.BlockRowsArgs(empty, empty, P, 2))[0] == hero.OK
    assert call("hero_block_cache_append", _cache(B=0), hero.BlockRowsArgs(_t(4, 256), _t(4, 256), P, 2))[0] == hero.OK
    q = _t(0, 512, data=None)
    assert call("hero_block_attention", _cache(), hero.BlockAttnArgs(q, q, P, 2, 4, 0.0, None, 0))[0] == hero.OK
    assert call("hero_qk_norm_rope", _rope(q=_t(0, 512, data=None), k=empty, q_out=q, k_out=empty))[0] == hero.OK


@pytest.mark.parametrize("kw", [dict(nq=3), dict(nq=1), dict(max_rows=0), dict(q=_t(4, 512, hero.I8)), dict(q=_t(4, 500)), dict(out=_t(3, 512)),
                                dict(out=_t(4, 512, hero.F32)), dict(out=_t(4, 512, hero.I8)), dict(out=_t(4, 512, hero.I8, 1, P)),
                                dict(scale=float("nan")), dict(scale=float("inf")), dict(row_start=None), dict(q=_t(4, 512, data=P + 4))])
def test_bad_attention_arguments_are_refused(call, kw):
    d = dict(q=_t(4, 512), out=_t(4, 512), row_start=P, max_rows=2, nq=4, scale=0.0, workspace=P, workspace_bytes=1 << 30)
    d.update(kw)
    assert call("hero_block_attention", _cache(), hero.BlockAttnArgs(**d))[0] not in (hero.OK, hero.ERR_CUDA)


@pytest.mark.parametrize("max_rows,nq", [(1 << 30, 4), ((1 << 31) - 1, 4), (1 << 24, 256)])
def test_a_row_bound_beyond_32_bit_row_numbers_is_refused(call, max_rows, nq):
    # rows of a key / value head are numbered (row of the sequence, query head of the group): 2^30 of them at most
    q = _t(4, nq * 128)
    args = hero.BlockAttnArgs(q, q, P, max_rows, nq, 0.0, P, 1 << 30)
    assert call("hero_block_attention", _cache(), args)[0] == hero.ERR_UNSUPPORTED
    n = C.c_size_t()
    blank = (C.c_uint8 * (1 << 20))()
    assert hero.lib().hero_block_attention_workspace_bytes(C.cast(blank, C.c_void_p), C.byref(_cache()), nq, 4, max_rows, C.byref(n)) == hero.ERR_UNSUPPORTED


def _rope(**kw):
    d = dict(q=_t(4, 512), k=_t(4, 256), q_out=_t(4, 512, data=2 * P), k_out=_t(4, 256, data=2 * P), nq=4, nkv=2, dh=128, rot=128, pairing=0,
             eps=1e-6, q_gamma=P, k_gamma=P, pos=P, cos=P, sin=P, n_pos=8)
    d.update(kw)
    return hero.QkNormRopeArgs(**d)


@pytest.mark.parametrize("kw", [dict(dh=120), dict(dh=272), dict(rot=8), dict(rot=144), dict(nq=0), dict(nkv=0), dict(pairing=2), dict(pos=None),
                                dict(cos=None), dict(n_pos=0), dict(sin=P + 4), dict(q=_t(4, 512, hero.F32)), dict(k=_t(4, 256, hero.F16)),
                                dict(k=_t(3, 256)), dict(q_out=_t(4, 512, hero.F16, data=2 * P)), dict(q_out=_t(4, 512, hero.I8, 2, P, data=2 * P)),
                                dict(q_out=_t(4, 512, hero.I8, 3, None, data=2 * P)), dict(q_out=_t(4, 512, hero.I8, 3, P)),
                                dict(q_out=_t(4, 512, ld=520)), dict(q=_t(4, 512, data=P + 8))])
def test_bad_rotation_arguments_are_refused(call, kw):
    assert call("hero_qk_norm_rope", _rope(**kw))[0] not in (hero.OK, hero.ERR_CUDA)


def test_struct_sizes_match_the_compiler():
    # x86-64 SysV sizes of the header's structs, field by field
    assert C.sizeof(hero.BlockCache) == 4 * 8 + 2 * 4 + 4 * 8 + 3 * 8 + 4 * 4
    assert C.sizeof(hero.BlockRowsArgs) == 2 * 48 + 8 + 8
    assert C.sizeof(hero.BlockAttnArgs) == 2 * 48 + 8 + 4 * 4 + 8 + 8      # the float is followed by 4 bytes of padding
    assert C.sizeof(hero.QkNormRopeArgs) == 4 * 48 + 6 * 4 + 6 * 8
