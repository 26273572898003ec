"""Layers whose tokens are in 8-bit caches only: made without pools, they give what layers with pools beside the cache give, and refuse what needs pools."""
import numpy as np
import pytest

import workloads as W
from tree_util import random_tree

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
CODES = pytest.mark.parametrize("code", [0, 1], ids=["int8", "e4m3"])
P, PAGES, H, H_KV, D = 16, 64, 8, 2, 64


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


def decode_layer(dtype, table, pools=None):
    from paper_2411_02886_amd.runtime import DecodeLayer
    ind, pages, lens = table
    return DecodeLayer(dtype=dtype, H=H, H_kv=H_KV, D=D, P=P, k=8, k_pool=pools, v_pool=pools, page_indptr=ind, page_indices=pages, seq_lens=lens, max_seq_len=400)


def chunk_layer(table, C, pools=None):
    from paper_2411_02886_amd.runtime import ChunkSelector
    ind, pages, lens = table
    return ChunkSelector(C=C, H=H, H_kv=H_KV, D=D, P=P, k=8, k_pool=pools, v_pool=pools, page_indptr=ind, page_indices=pages, seq_lens=lens, max_seq_len=400)


def serve(ts, dtype, code, pools):
    """Two prompts, one of them in chunks and forked, then a tree of each, its path, and a token behind it: everything that comes out."""
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import copy_pages
    rng, pool = np.random.default_rng(code), PagePool(PAGES, P)
    cache = ts.QuantCache.empty(PAGES, P, H_KV, D, code)
    stored = torch.int16 if dtype == BF else torch.float32
    rope = ts.Rope(inv_freq=dev((1e4 ** -(np.arange(16) / 16)).astype(np.float32)))
    rows = lambda n, h: dev(W.store(rng.standard_normal((n, h, D), dtype=np.float32), dtype))
    zeros = lambda n: (torch.zeros((n, H, D), dtype=stored, device="cuda:0"), torch.zeros((n, H), device="cuda:0"))
    got = []

    def call(lay, new, mask=None, pos=None, packed=True, most=None):
        T = sum(new)
        ind = dev(np.cumsum([0] + new).astype(np.int32)) if packed else None
        q, (out, lse) = zeros(T)[0], zeros(T)
        lay.append(rows(T, H_KV), rows(T, H_KV), q=rows(T, H), q_out=q, rope=rope, positions=pos, q_indptr=ind, cache=cache)
        lay.attend_all(q, q_indptr=ind, out=out, lse=lse, most_new=most, mask=mask, cache=cache)
        got.extend((q, out, lse))

    for s, parts in (("a", [37]), ("b", [30, 60])):
        pool.add(s)
        for n in parts:
            pool.grow(s, n)
            lay = chunk_layer(pool.table([s]), n, pools) if dtype == BF else decode_layer(dtype, pool.table([s]), pools)
            call(lay, [n], packed=dtype != BF, most=n)
    pool.fork("b", "c")
    seqs, new = ["a", "b", "c"], [9, 1, 40]
    for s, n in zip(seqs, new):
        copies = pool.grow(s, n)
        copy_pages(decode_layer(dtype, pool.table([s]), pools).problem, copies, PAGES, cache=cache)
    lay, T = decode_layer(dtype, pool.table(seqs), pools), sum(new)
    mask, pos = torch.zeros((T, 2), dtype=torch.int32, device="cuda:0"), torch.zeros((1, T), dtype=torch.int32, device="cuda:0")
    ind = dev(np.cumsum([0] + new).astype(np.int32))
    lay.tree_mask(dev(np.concatenate([random_tree(rng, n) for n in new])), mask, positions=pos, q_indptr=ind)
    call(lay, new, mask=mask, pos=pos, most=max(new))
    to_lens = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    lay.keep(dev(np.array([[0, 4, 8], [0, 0, 0], [0, 1, 30]], np.int32)), dev(np.array([3, 0, 2], np.int32)), to_lens, q_indptr=ind, cache=cache)
    for s, n in zip(seqs, to_lens.tolist()):
        pool.cut(s, n)
        pool.grow(s, 1)                                  # (their last pages are their own since the drafts)
    lay = decode_layer(dtype, pool.table(seqs), pools)
    call(lay, [1, 1, 1], packed=False)
    lens = lay.seq_lens.tolist()
    back = [torch.zeros((sum(lens), H_KV, D), dtype=stored, device="cuda:0") for _ in "kv"]
    lay.read_back(cache, *back, q_indptr=dev(np.cumsum([0] + lens).astype(np.int32)))
    torch.cuda.synchronize()
    return got + [mask, pos, to_lens] + back + list(cache._keep), lay


@DTYPES
@CODES
def test_a_layer_needs_no_pools_beside_its_cache(gpu, dtype, code):
    pools = torch.zeros((PAGES, P, H_KV, D), dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0")
    with_pools, _ = serve(gpu, dtype, code, pools)
    without, lay = serve(gpu, dtype, code, None)
    assert lay.k_pool is None and lay.v_pool is None and len(without) == len(with_pools)
    for i, (a, b) in enumerate(zip(with_pools, without)):
        assert torch.equal(a, b), i
    assert not pools.any() and all(x.any() for x in without[:15])


def test_a_captured_step_without_pools(gpu):
    from paper_2411_02886_amd.pages import PagePool
    pool = PagePool(PAGES, P)
    for s, n in (("a", 30), ("b", 100)):
        pool.add(s, n)
    cache = gpu.QuantCache.empty(PAGES, P, H_KV, D, 0)
    lay = decode_layer(BF, pool.table(["a", "b"], room=2))
    rng = np.random.default_rng(0)
    k, v, q = (dev(W.store(rng.standard_normal((130, h, D), dtype=np.float32), BF)) for h in (H_KV, H_KV, H))
    lay.append(k, v, q_indptr=dev(np.array([0, 30, 130], np.int32)), cache=cache)
    step = [t[:2].contiguous() for t in (k, v, q)]

    def one():
        lay.seq_lens.add_(1)
        lay.append(step[0], step[1], cache=cache)
        lay.attend_all(step[2], cache=cache)

    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        one()                                            # (the layer makes its workspace)
        lay.seq_lens.sub_(1)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        one()
    for rep in range(4):
        start = lay.seq_lens.clone()
        graph.replay()
        torch.cuda.synchronize()
        got = lay.out.clone(), lay.lse.clone(), lay.seq_lens.clone()
        lay.seq_lens.copy_(start)
        lay.out.zero_()
        one()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (lay.out, lay.lse, lay.seq_lens))) and got[0].any(), rep


def test_what_needs_pools_is_refused_and_changes_nothing(gpu):
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import copy_pages
    pool = PagePool(PAGES, P)
    pool.add("a", 30)
    lay, chunk = decode_layer(BF, pool.table(["a"])), chunk_layer(pool.table(["a"]), 4)
    q, kv = torch.ones((1, 1, H, D), dtype=torch.int16, device="cuda:0"), torch.zeros((1, H_KV, D), dtype=torch.int16, device="cuda:0")
    z = torch.zeros(2, dtype=torch.int32, device="cuda:0")
    calls = [lambda: lay.append(kv, kv), lambda: lay.attend_all(q), lambda: lay.attend_all(q, mask=z.view(1, 2)[:, :1].contiguous()),
             lambda: lay.attend_all(q, round_weights=True), lambda: lay.keep(z.view(1, 2), z[:1], z[1:]), lambda: lay.select(q),
             lambda: lay.select_compact(q), lambda: lay.attend(q, 0.1), lambda: lay.step(q), lambda: lay.step(q, theta=0.9), lambda: lay.step(q, compact=True),
             lambda: lay.step(q, theta=0.9, compact=None, fused_check=True), lambda: lay.compact(z, z, z), lambda: chunk.select(q), lambda: chunk.attend(q),
             lambda: chunk.select_mean_query(q), lambda: copy_pages(lay.problem, [(0, 1)], PAGES),
             lambda: copy_pages(lay.problem, [(0, 1)], PAGES, device="cuda:0"), lambda: lay.swap_pool(kv, None)]
    for i, call in enumerate(calls):
        with pytest.raises(ValueError):
            call()
            assert False, i
    torch.cuda.synchronize()
    assert lay.first.all() and not lay.cached_q.any() and not lay.reuse.any() and not lay.out.any() and lay.k_pool is None
    q_out = torch.zeros((1, H, D), dtype=torch.int16, device="cuda:0")
    lay.append(None, None, q=q, q_out=q_out)             # queries alone need no pools
    torch.cuda.synchronize()
    assert torch.equal(q_out.flatten(), q.flatten())
    for make in (lambda p: decode_layer(BF, pool.table(["a"]), p), lambda p: chunk_layer(pool.table(["a"]), 4, p)):
        make(None)
    with pytest.raises(ValueError):
        from paper_2411_02886_amd.runtime import DecodeLayer
        ind, pages, lens = pool.table(["a"])
        DecodeLayer(dtype=BF, H=H, H_kv=H_KV, D=D, P=P, k=8, k_pool=kv, v_pool=None, page_indptr=ind, page_indices=pages, seq_lens=lens)
