"""ts_tree_mask refuses results that lie in what its other workgroups still read, before anything is launched."""
import ctypes

import pytest

import paper_2411_02886_amd as ts
from paper_2411_02886_amd.binding import _CProblem

B, T, WORDS = 3, 50, 2
PARENTS, LENS, INDPTR, MASK, POSITIONS = (0x100000 * i for i in range(1, 6))


def call(**kw):
    a = dict(parents=PARENTS, ind=INDPTR, mask=MASK, pos=POSITIONS, lens=LENS)
    a.update(kw)
    p = _CProblem(batch=B, chunk=1, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=4096, dtype=ts.TS_BF16, k_pool=None, v_pool=None,
                  page_indptr=0x10000, page_indices=0x10000, seq_lens=a["lens"], num_initial=0, num_local=0)
    return ts.load().ts_tree_mask(ctypes.byref(p), a["parents"], a["ind"], T, a["mask"], WORDS, a["pos"], None)


@pytest.mark.parametrize("name,at,size", [("parents", PARENTS, T * 4), ("lens", LENS, B * 4), ("ind", INDPTR, (B + 1) * 4)], ids=lambda x: x if isinstance(x, str) else "")
def test_results_over_what_is_read(name, at, size):
    for what, room in (("mask", T * WORDS * 4), ("pos", T * 4)):
        for place in (at, at + size - 4, at - room + 4):
            assert call(**{what: place}) == -1, (what, place - at)


def test_positions_over_the_mask():
    for place in (MASK, MASK + T * WORDS * 4 - 4, MASK - T * 4 + 4):
        assert call(pos=place) == -1
