"""The cache's calls as the layers offer them: lists of copies, shapes, workspaces, streams."""
import numpy as np
import pytest

import workloads as W
from cache_util import Cache, attention, check_attention

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def test_joined_lists_of_page_copies_are_made_in_their_order(gpu):
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import copy_pages
    P, NP = 256, 64
    k = torch.arange(NP, dtype=torch.int32, device="cuda:0")[:, None, None, None].repeat(1, P, 2, 64)
    v = -k
    z = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    p = gpu.Problem(batch=1, num_q_heads=2, num_kv_heads=2, head_dim=64, page_size=P, max_seq_len=1, dtype=F32, k_pool=k, v_pool=v, page_indptr=z,
                    page_indices=z, seq_lens=z)
    pool, copies = PagePool(NP, P), []
    pool.add(0, 3)
    for i in range(NP - 1):                              # each child forks the one before and grows: a chain of copies
        pool.fork(i, i + 1)
        copies += pool.grow(i + 1)
    assert copies == [(i, i + 1) for i in range(NP - 1)]
    copy_pages(p, copies, NP)
    torch.cuda.synchronize()
    assert not k.any() and not v.any()
