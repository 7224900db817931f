"""The oracle's append: what becomes of a page's scale.  A partly filled page's never shrinks and is the larger of the old one and what the new
tokens call for; a page that is begun takes it from the new tokens alone, whatever it held before."""
import numpy as np
import pytest

from oracle import block_cache as BC


@pytest.mark.parametrize("kind", ["i8", "f8"])
def test_scales_of_partly_filled_pages_grow_only_and_begun_pages_forget(kind):
    g = np.random.default_rng(7)
    pages, heads, page, dh = 5, 2, 16, 64
    c, s = np.zeros((pages, heads, page, dh)), np.full((pages, heads), 9.0, np.float32)
    table = [3, 1, 0]
    x = (g.standard_normal((40, heads * dh)) * np.exp(g.standard_normal((40, 1)))).astype(np.float32)
    at, kept, grown = 0, 0, 0
    for n in (1, 4, 20, 1, 2, 12):                         # 40 tokens, over page borders
        new = x[at:at + n].reshape(n, heads, dh)
        c2, s2 = BC.append(c, s, [table], [at + n], [n], [0], x[at:at + n], page, kind)
        for pi, pid in enumerate(table):
            lo, hi = max(at - pi * page, 0), min(at + n - pi * page, page)         # slots that receive tokens
            if hi <= lo:
                assert np.array_equal(s2[pid], s[pid]) and np.array_equal(c2[pid], c[pid])
                continue
            rows = new[pi * page + lo - at:pi * page + hi - at]
            asked = np.abs(rows).max((0, 2)) / np.float32(BC.top(kind))
            assert asked.dtype == np.float32
            if lo == 0:
                assert np.array_equal(s2[pid], asked)
            else:
                assert np.all(s2[pid] >= s[pid]) and np.array_equal(s2[pid], np.maximum(s[pid], asked))
                same = s2[pid] == s[pid]
                assert np.array_equal(c2[pid][same, :lo], c[pid][same, :lo])       # an unchanged scale leaves the codes alone
                kept, grown = kept + same.sum(), grown + (~same).sum()
        c, s = c2, s2
        at += n
    assert kept and grown                                  # both cases were met
