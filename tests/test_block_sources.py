"""Kernels of the block cache may be resident while the kernel before them still runs, so only what no call of the stream writes may be
read through the non-coherent path: gammas, rotation tables and output scales (model constants)."""
import os
import re

import pytest

from paper_2310_17723_b200 import build as B

FILES = ["block_cache.cuh", "block_cache.cu", "block_attention.cuh", "block_attention.cu", "block_attention_prompt.cu", "qk_rope.cu"]
CONSTANTS = re.compile(r"^(p\.out_scale\b|p\.cos\b|p\.sin\b|gm\b)")


@pytest.mark.parametrize("name", FILES)
def test_only_constants_are_read_through_the_non_coherent_path(name):
    with open(os.path.join(B.CSRC, name)) as f:
        text = re.sub(r"//.*", "", f.read())
    assert not re.search(r"ld\.global\.nc|__restrict__", text)
    for m in re.finditer(r"__ldg\(", text):
        assert CONSTANTS.match(text[m.end():]), text[m.start():m.end() + 40]
