"""hero_block_attention_workspace_bytes on sizes at the edge of what is taken, without a GPU (a blank handle: no SMs)."""
import ctypes as C

from paper_2310_17723_b200 import build as B
from paper_2310_17723_b200 import hero


def test_a_smaller_row_bound_that_is_refused_does_not_refuse_the_one_asked_for():
    # 65535 sequences x 16384 heads: 33 rows are one tile of 256 rows each, 28 would be two tiles of 16 and more groups than are numbered
    B.build()
    blank = (C.c_uint8 * (1 << 20))()
    p = 1 << 20
    cache = hero.BlockCache(p, p, p, p, hero.I8, 64, 10, 64 * 64 * 16384, 64 * 64, 64, p, 4, p, 256, 65535, 16384, 64)
    n = C.c_size_t()
    ask = lambda rows: hero.lib().hero_block_attention_workspace_bytes(C.cast(blank, C.c_void_p), C.byref(cache), 16384, 4, rows, C.byref(n))  # noqa: E731
    assert ask(28) == hero.ERR_UNSUPPORTED
    assert ask(33) == hero.OK and n.value == 0
    assert ask(8) == hero.OK
