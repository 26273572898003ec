"""Attention whose sequences have up to 128 rows on average (new tokens times query heads of a KV head), where the halves of a workgroup have half of a tile's
keys each: against the definition in 64 bits, over 8-bit caches and, for trees, bf16 pools.  One half may see no key of a row, or none at all."""
import numpy as np
import pytest

import workloads as W
from cache_util import Cache, check_attention
from quant_util import QuantPages
from test_gpu_quant_attn import run as run_quant, trees
from test_gpu_tree import run as run_tree

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF = W.BF16
KINDS = pytest.mark.parametrize("kind", [0, 1, None], ids=["int8", "e4m3", "pools"])
SHAPES = pytest.mark.parametrize("H,H_kv,D", [(28, 4, 128), (32, 8, 128), (8, 1, 64), (10, 2, 64)])


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def check(ts, kind, H, H_kv, D, new, lens, tree, **kw):
    sees = trees(new, H + D, roots=True) if tree else None
    if kind is None:
        c = Cache(BF, H_kv, D, 16, lens, seed=H)
        sees = [np.tril(np.ones((n, n), dtype=bool)) for n in new] if sees is None else sees
        got = run_tree(ts, c, H, new, sees, seed=H, **kw)
    else:
        c = QuantPages(BF, kind, H_kv, D, 16, lens, seed=H)
        got = run_quant(ts, c, H, new, seed=H, sees=sees, **kw)
    check_attention(*got, (kind, new, lens))


# 65 to 128 rows; keys of less than half a tile, of one, of one and a half, and of many
@KINDS
@SHAPES
@pytest.mark.parametrize("rows", [65, 96, 97, 128])
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_rows_and_keys(gpu, kind, H, H_kv, D, rows, tree):
    n = max(64 // (H // H_kv) + 1, rows // (H // H_kv))
    check(gpu, kind, H, H_kv, D, [n] * 7, [n, n + 1, n + 15, n + 40, n + 64, n + 97, n + 700], tree, packed=False)


# sequences of one token to three tiles side by side, some without new tokens, one with fewer tokens than new ones
@KINDS
@SHAPES
@pytest.mark.parametrize("loose", [False, True], ids=["", "loose bound"])
def test_mixed_batches_in_shares(gpu, kind, H, H_kv, D, loose):
    n = 128 // (H // H_kv)
    new = [n, 1, 3, 2 * n + 5, 0, n - 1, 9]
    lens = [7000 + n, 300, 3, 9000, 40, 2500, 5]
    check(gpu, kind, H, H_kv, D, new, lens, True, behind=3, max_seq_len=300000 if loose else None)


@KINDS
@pytest.mark.parametrize("window", [1, 31, 32, 33, 64, 65, 100, 3000])
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_windows(gpu, kind, window, tree):
    if kind is None and not tree:
        pytest.skip("causal windows over pools are another call")
    new = [18, 10, 17, 11]
    check(gpu, kind, 28, 4, 128, new, [18, 4000, 90, 600], tree, window=window)


# Large and small logits: the halves' references differ by far more than float's exponents reach.
@KINDS
@pytest.mark.parametrize("sm,q_scale", [(0.0, 1.0), (-0.3, 1.0), (64.0, 30.0)])
def test_references_far_apart(gpu, kind, sm, q_scale):
    check(gpu, kind, 8, 1, 64, [12, 16], [1200, 90], True, sm=sm, q_scale=q_scale)


# Nothing but one half's keys: a row sees a single new token beside it and no cached one.
@KINDS
@pytest.mark.parametrize("base", [0, 31, 32, 63, 64, 95])
def test_one_half_sees_nothing(gpu, kind, base):
    n, H, H_kv, D = 16, 8, 1, 64
    sees = [np.eye(n, dtype=bool)]
    sees[0][3] = False                                   # and this row sees nothing at all
    kw = dict(window=1, packed=False, seed=base)
    if kind is None:
        got = run_tree(gpu, Cache(BF, H_kv, D, 16, [base + n], seed=base), H, [n], sees, **kw)
    else:
        got = run_quant(gpu, QuantPages(BF, kind, H_kv, D, 16, [base + n], seed=base), H, [n], sees=sees, **kw)
    check_attention(*got, base)


@KINDS
def test_the_same_call_gives_the_same_bits(gpu, kind):
    new, lens = [18, 14, 16], [9000, 300, 4000]
    both = []
    for _ in range(2):
        if kind is None:
            both.append(run_tree(gpu, Cache(BF, 4, 128, 16, lens, seed=1), 28, new, trees(new, 1), seed=1)[:2])
        else:
            both.append(run_quant(gpu, QuantPages(BF, kind, 4, 128, 16, lens, seed=1), 28, new, seed=1, sees=trees(new, 1))[:2])
    assert np.array_equal(both[0][0], both[1][0]) and np.array_equal(both[0][1], both[1][1])
