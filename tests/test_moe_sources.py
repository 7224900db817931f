"""What the epilogue of the grouped products does when a wait gives up cannot be made to happen from outside; its order is read here: all warps of a group have their
vectors and products, or the group writes nothing of the tile and leaves."""
import os
import re

from paper_2310_17723_b200 import build as B


def test_no_warp_of_a_group_writes_before_all_have_what_they_waited_for():
    with open(os.path.join(B.CSRC, "moe_linear.cu")) as f:
        text = re.sub(r"//.*", "", f.read())
    body = text[text.index("void moe_epilogue("):]
    body = body[body.index("for (int it = 0;; ++it)"):body.index("moe_linear_body(")]
    vectors, products = body.index("mbar_wait(&vec_full"), body.index("mbar_wait(&acc_full")
    agreed = body.index("group_all(")
    assert vectors < products < agreed < min(body.index(n) for n in ("moe_tmem_ld", "moe_chunk", "moe_store", "atomicMax", "mbar_arrive"))
    assert re.search(r"if \(!group_all\(ok, 1 \+ group\)[^;]*\) break;", body)
    assert body.count("mbar_wait(") == 2 and body.count("group_all(") == 1
    assert not re.search(r"\bok\b", body[agreed + len("group_all(ok"):])      # nothing goes on with half of it
