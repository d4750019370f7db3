"""Room that the attention over a 4-bit cache asks for: logits of the heads that there are, partial results of as many units and pieces as a
launch has (no GPU needed)."""

import ctypes

import pytest

from paper_2506_02850_b200 import binding as B
from paper_2506_02850_b200 import build as builder


@pytest.fixture(scope="module")
def lib():
    builder.build()
    return B.lib()


@pytest.mark.parametrize("dtype", [B.BF16, B.F32])
@pytest.mark.parametrize("Hq,Hkv,dh,n_seqs,page,max_pages", [(40, 40, 128, 48, 16, 563), (28, 4, 128, 3, 64, 290), (14, 2, 64, 5, 32, 40), (33, 1, 64, 1, 16, 1),
                                                             (36, 2, 128, 7, 256, 30), (2048, 1, 64, 1, 16, 9), (3, 3, 64, 300, 16, 3)])
def test_room_for_the_heads_that_there_are(lib, dtype, Hq, Hkv, dh, n_seqs, page, max_pages):
    c = B.PagedCache(None, None, None, None, 4096, Hkv, page, dh, n_seqs, max_pages)
    size = lambda mass: lib.metok_paged_attention_q4_workspace_bytes(dtype, ctypes.byref(c), Hq, mass)
    G = Hq // Hkv
    units = Hkv * -(-G // 16)                                        # of a sequence: of at most sixteen heads, of each of which one may be missing
    heads = Hq + units
    rows = -(-max_pages * page // 128) * 128                         # whole tiles
    pieces = 3 * 148
    partials = 4 * (dh + 2) * (n_seqs * heads + pieces * (-(-G // -(-G // 16)))) + 8 * (n_seqs + 1)
    assert 0 < size(0) <= partials + 4 * 256
    assert 4 * n_seqs * Hq * rows <= size(1) - size(0) <= 4 * n_seqs * heads * rows + 256
