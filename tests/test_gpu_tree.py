"""ts_tree_mask, ts_tree_attn and ts_tree_keep: masks from parents, attention with masks of trees and of any bits against the definition in 64 bits, accepted
paths moved behind the cached tokens, and the three together as a step of speculative decoding."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache, check_attention
from quant_util import QuantPages
from tree_util import attention, closure, random_tree, words_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def dev(x):
    from paper_2411_02886_amd.runtime import to_device
    return to_device(x)


def indptr(new):
    return dev(np.cumsum([0] + list(new)).astype(np.int32))


def masks(ts, parents, new, lens, words, packed=True, behind=0, positions=True):
    z = dev(np.zeros(len(new) + 1, np.int32))
    p = ts.Problem(batch=len(new), chunk=max(1, max(new)), num_q_heads=1, num_kv_heads=1, head_dim=64, page_size=16, max_seq_len=1 << 20, dtype=F32,
                   k_pool=None, v_pool=None, page_indptr=z, page_indices=z, seq_lens=dev(np.asarray(lens, np.int32)))
    T = sum(new) + behind
    mask = torch.full((T, words), 77, dtype=torch.int32, device="cuda:0")
    pos = torch.full((T,), 77, dtype=torch.int32, device="cuda:0") if positions else None
    par = np.concatenate([*parents, np.zeros(behind, np.int32)]).astype(np.int32)
    ts.ts_tree_mask(p, dev(par), indptr(new) if packed else None, T, mask, pos)
    torch.cuda.synchronize()
    return mask.cpu().numpy().view(np.uint32), None if pos is None else pos.cpu().numpy()


@pytest.mark.parametrize("words", [1, 2, 3, 8, 40])
@pytest.mark.parametrize("packed", [True, False], ids=["packed", "padded"])
def test_masks_of_trees(gpu, words, packed):
    rng = np.random.default_rng(words)
    new = [33, 1, 0, 64, 65, 200, 7, 1000] if packed else [70] * 6
    lens = [n + int(rng.integers(0, 500)) for n in new]
    lens[1] = 0                                              # fewer tokens than new ones: a negative place
    parents = [random_tree(rng, n, near=1 + 7 * (b % 3), roots=b % 2 == 1) for b, n in enumerate(new)]
    got, pos = masks(gpu, parents, new, lens, words, packed, behind=3 if packed else 0)
    row = 0
    for n, N, par in zip(new, lens, parents):
        sees = closure(par)
        if n:
            assert np.array_equal(got[row:row + n], words_of(sees, words)), n
            assert np.array_equal(pos[row:row + n], N - n + sees.sum(axis=1) - 1), n
        row += n
    assert np.all(got[row:] == 77) and np.all(pos[row:] == 77)


def test_what_cannot_be_a_parent_makes_a_root_and_long_chains(gpu):
    n = 5000                                                 # more than are staged, one path through all of them
    chain = np.arange(-1, n - 1, dtype=np.int32)
    odd = np.array([0, 5, -7, 2, 4, 1 << 30, -(1 << 31), 3, 2], np.int32)
    got, _ = masks(gpu, [chain, odd], [n, len(odd)], [n, len(odd)], (n + 31) // 32, positions=False)
    assert np.array_equal(got[:n], words_of(np.tril(np.ones((n, n), bool)), (n + 31) // 32))
    assert np.array_equal(got[n:], words_of(closure(odd), (n + 31) // 32))


def run(ts, cache, H, new, sees, window=0, packed=True, sm=None, seed=0, max_seq_len=None, behind=0, chunk=None, words=None, q_scale=1.0, q=None):
    from paper_2411_02886_amd.runtime import to_host
    D, T = cache.D, sum(new) + behind
    sm = 1.0 / math.sqrt(D) if sm is None else sm
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    q = W.store(q_scale * rng.standard_normal((T, H, D), dtype=np.float32), cache.dtype) if q is None else q
    p = cache.problem(H, chunk=max(1, max(new)) if chunk is None else chunk, max_seq_len=max_seq_len)[0]
    words = max(1, (max(new) + 31) // 32) if words is None else words
    mask = np.concatenate([words_of(s, words) for s in sees if len(s)] + [np.zeros((behind, words), np.uint32)])
    es = torch.int16 if cache.dtype == BF else torch.float32
    out = torch.full((T, H, D), 77, dtype=es, device="cuda:0")
    lse = torch.full((T, H), 55.0, dtype=torch.float32, device="cuda:0")
    n = ts.ts_paged_attn_workspace_bytes(p, T)
    ws = torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")
    ts.ts_tree_attn(p, dev(q), indptr(new) if packed else None, T, window, dev(mask.view(np.int32)), sm, out, lse, ws)
    torch.cuda.synchronize()
    o, l = to_host(out, bits16=cache.dtype == BF), to_host(lse)
    if behind:
        assert np.all(o[T - behind:] == 77) and np.all(l[T - behind:] == 55.0)
    seen = [s & (np.arange(len(s)) < 32 * words) for s in sees]
    ref = attention(cache, q[:T - behind], new, window, float(np.float32(sm)), seen)
    return W.as_f32(o, cache.dtype).astype(np.float64)[:T - behind], l[:T - behind].astype(np.float64), ref


def trees(new, seed, **kw):
    rng = np.random.default_rng(seed)
    return [closure(random_tree(rng, n, **kw)) for n in new]


HEADS = [(1, 1), (8, 8), (8, 4), (6, 2), (8, 2), (10, 2), (6, 1), (28, 4), (16, 2), (32, 32)]


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_trees_of_every_head_layout(gpu, dtype, D, H, H_kv):
    new, old = [13, 1, 40, 65], [0, 300, 129, 31]
    c = Cache(dtype, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H * 17 + D)
    check_attention(*run(gpu, c, H, new, trees(new, H), seed=H), "trees")


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 5, 16, 31, 32, 33, 63, 64, 65, 96, 130, 257])
def test_sizes_of_a_tree(gpu, dtype, D, n):
    c = Cache(dtype, 2, D, 16, [n, n + 1, n + 31, n + 63, n + 64, n + 200], seed=n)
    check_attention(*run(gpu, c, 8, [n] * 6, trees([n] * 6, n, roots=True), packed=False, seed=n), n)


@DTYPES
@pytest.mark.parametrize("window", [1, 2, 15, 63, 64, 65, 100, 128, 1 << 30])
@pytest.mark.parametrize("D", [64, 128])
def test_windows(gpu, dtype, window, D):
    new = [1, 90, 0, 5, 64]
    c = Cache(dtype, 2, D, 8, [300, 290, 17, 5, 517], seed=window % 1000)
    check_attention(*run(gpu, c, 6, new, trees(new, 3), window=window, seed=3), window)


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [9, 40, 150])
def test_any_bits(gpu, dtype, D, n):
    """Rows that see later tokens, all of them, not themselves, nothing; fewer words than tokens."""
    rng = np.random.default_rng(n)
    for old in (0, 1, 70):
        sees = [rng.random((n, n)) < 0.3, np.ones((n, n), bool), np.zeros((n, n), bool)]
        sees[0][n // 2] = False
        sees[0][:, n - 2] = False
        c = Cache(dtype, 2, D, 16, [n + old] * 3, seed=n + old)
        for words in (None, 1, 9):
            o, l, ref = run(gpu, c, 8, [n] * 3, sees, seed=n, words=words)
            check_attention(o, l, ref, (old, words))
        assert old or np.isneginf(l[2 * n:]).all()


@DTYPES
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_without_tokens_and_rows_that_see_nothing(gpu, dtype, D):
    new, lens = [0, 3, 70, 2, 0, 1, 40], [0, 0, 30, 2, 9, 0, 41]
    c = Cache(dtype, 4, D, 16, lens, seed=5)
    check_attention(*run(gpu, c, 8, new, trees(new, 5), seed=5, behind=3), "empty")


@DTYPES
def test_a_chain_gives_what_dense_attention_gives(gpu, dtype):
    """A tree without branches is a draft: the causal mask, which ts_paged_attn computes."""
    from paper_2411_02886_amd.runtime import to_host
    new = [5, 40, 1, 100]
    c = Cache(dtype, 2, 128, 16, [n + 500 for n in new], seed=2)
    o, l, ref = run(gpu, c, 8, new, [np.tril(np.ones((n, n), bool)) for n in new], seed=2)
    check_attention(o, l, ref, "chain")
    dense = attention(c, W.store(np.random.Generator(np.random.PCG64(1002)).standard_normal((sum(new), 8, 128), dtype=np.float32), dtype), new, 0,
                      float(np.float32(1 / math.sqrt(128))))
    check_attention(o, l, dense, "dense")


@pytest.mark.parametrize("dtype,H,H_kv,D,new,old", [(BF, 32, 8, 128, [60, 3, 64], [9000, 20001, 5]), (F32, 8, 2, 64, [13, 40], [6000, 11000]),
                                                    (BF, 4, 4, 64, [7], [12345]), (BF, 16, 4, 128, [200, 1], [5001, 70]), (BF, 8, 1, 64, [64], [20000])])
@pytest.mark.parametrize("loose", [False, True], ids=["", "loose bound"])
@pytest.mark.parametrize("window", [0, 3000])
def test_long_caches_are_cut_into_shares(gpu, dtype, H, H_kv, D, new, old, loose, window):
    lens = [a + b for a, b in zip(new, old)]
    c = Cache(dtype, H_kv, D, 16, lens, seed=H)
    check_attention(*run(gpu, c, H, new, trees(new, H), seed=H, window=window, max_seq_len=300000 if loose else None, chunk=200 if loose else None), lens)


@DTYPES
@pytest.mark.parametrize("sm,q_scale", [(0.0, 1.0), (-0.3, 1.0), (64.0, 30.0)])
@pytest.mark.parametrize("n", [6, 60])
def test_scales_and_large_logits(gpu, dtype, sm, q_scale, n):
    c = Cache(dtype, 2, 64, 16, [n + 150, n + 40], seed=n, scale=q_scale)
    check_attention(*run(gpu, c, 8, [n] * 2, trees([n] * 2, n), packed=False, sm=sm, q_scale=q_scale, seed=n), (sm, q_scale))


@DTYPES
@pytest.mark.parametrize("n", [6, 60, 100])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_keys_that_a_row_does_not_see_may_be_anything(gpu, dtype, n, bad):
    """K of a node that only its own row sees, which comes out NaN; every other row as if it were not there."""
    c = Cache(dtype, 2, 64, 16, [n + 90], seed=n)
    sees = np.eye(n, dtype=bool) | (np.arange(n) == 0)
    s = c.slots(0)[90 + 3]
    bits = W.store(np.full((2, 64), bad, np.float32), dtype)
    c.k_bits[s] = np.full((2, 64), 0x7fc0, np.uint16) if dtype == BF and np.isnan(bad) else bits
    o, l, ref = run(gpu, c, 8, [n], [sees], seed=n)
    rest = np.arange(n) != 3
    check_attention(o[rest], l[rest], [x[rest] for x in ref], n)
    assert not np.isfinite(o[3]).any() or np.isinf(bad)


@pytest.mark.parametrize("quant", [None, 0, 1], ids=["plain", "int8", "e4m3"])
@pytest.mark.parametrize("dtype,H_kv,D,P", [(BF, 8, 128, 16), (F32, 32, 128, 8), (BF, 1, 64, 8), (F32, 2, 64, 1), (BF, 16, 64, 64)])
@pytest.mark.parametrize("packed", [True, False], ids=["packed", "padded"])
def test_keep(gpu, quant, dtype, H_kv, D, P, packed):
    rng = np.random.default_rng(P)
    new = [20, 1, 0, 64, 7, 150, 3] if packed else [30] * 7
    old = [0, 13, 5, 100, 77, 31, 9]
    lens = [a + b for a, b in zip(new, old)]
    lens[6] = 1                                              # fewer tokens than new ones
    stride = 80
    kept = [min(n, stride, int(rng.integers(0, n + 1))) for n in new]
    kept[3 if packed else 0], kept[4] = (64 if packed else 30), 0
    path = np.full((7, stride), -1, np.int32)
    for b, (m, n) in enumerate(zip(kept, new)):
        path[b, :m] = np.sort(rng.choice(n, m, replace=False))
    if packed:
        path[0, :4], kept[0] = [3, 3, 1, 500], 4             # an entry twice, one too small (it counts as its place), one too large
    count = np.array(kept, np.int32)
    count[5] += 1000                                         # clamped to the path's room, here with what follows -1: their own places
    kept[5] = min(stride, new[5])
    c = Cache(dtype, H_kv, D, P, lens, seed=P) if quant is None else QuantPages(dtype, quant, H_kv, D, P, lens, seed=P)
    held = c.problem(H_kv, chunk=max(new), max_seq_len=max(lens))
    p, q8 = held[0], None if quant is None else held[1]
    to_lens = torch.full((7,), -9, dtype=torch.int32, device="cuda:0")
    gpu.ts_tree_keep(p, q8, dev(path), stride, dev(count), indptr(new) if packed else None, to_lens)
    torch.cuda.synchronize()
    assert to_lens.cpu().tolist() == [max(0, N - n + m) for N, n, m in zip(lens, new, kept)]
    if quant is None:
        from paper_2411_02886_amd.runtime import to_host
        got = [to_host(t, bits16=dtype == BF).reshape(-1, H_kv, D) for t in held[1:]]
        want = [c.k_bits.reshape(-1, H_kv, D).copy(), c.v_bits.reshape(-1, H_kv, D).copy()]
    else:
        codes, scales = c.read(q8)
        got, want = [codes["k"], codes["v"], scales["k"], scales["v"]], [x.copy() for x in (c.bytes["k"], c.bytes["v"], c.scales["k"], c.scales["v"])]
    for b, (n, N) in enumerate(zip(new, lens)):
        at = c.slots(b)
        moved = [(N - n + i, N - n + min(max(int(path[b, i]), i), n - 1)) for i in range(kept[b])]
        for x in want:
            rows = {to: x[at[src]].copy() for to, src in moved if to >= 0}
            for to, row in rows.items():
                x[at[to]] = row
    for x, y in zip(got, want):
        view = {2: np.uint16, 4: np.uint32, 1: np.uint8}[x.dtype.itemsize]
        assert np.array_equal(np.ascontiguousarray(x).view(view), np.ascontiguousarray(y).view(view))


def test_keep_leaves_what_lies_beyond_the_bound(gpu):
    c = Cache(BF, 2, 64, 16, [40], seed=1)
    p, k, v = c.problem(2, chunk=20, max_seq_len=30)
    path, to = dev(np.array([[5, 8, 15]], np.int32)), torch.zeros(1, dtype=torch.int32, device="cuda:0")
    gpu.ts_tree_keep(p, None, path, 3, dev(np.array([3], np.int32)), None, to)
    torch.cuda.synchronize()
    want = c.k_bits.copy()
    at = c.slots(0)
    want[at[20]], want[at[21]] = c.k_bits[at[25]], c.k_bits[at[28]]          # place 35 is not read
    assert np.array_equal(k.cpu().numpy().view(np.uint16).reshape(want.shape), want) and to.item() == 23


def test_nothing_to_do(gpu):
    c = Cache(BF, 2, 64, 16, [5], seed=1)
    p, _, _ = c.problem(2)
    gpu.ts_tree_mask(p, None, None, 0, torch.zeros((1, 1), dtype=torch.int32, device="cuda:0"), None)
    gpu.ts_tree_attn(p, None, None, 0, 0, torch.zeros((1, 1), dtype=torch.int32, device="cuda:0"), 0.1, None, None, None)
    torch.cuda.synchronize()
