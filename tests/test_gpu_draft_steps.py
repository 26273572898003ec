"""Speculative decoding as a server runs it, through the layers: a prompt, a forked conversation, drafted trees that are masked, appended, attended and cut
down to an accepted path, and the next step behind it; over pools and over a cache in 8 bits, called and captured, and in pools beyond 4 GiB."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import check_attention
from quant_util import QuantPages, encode, of_code
from tree_util import attention, closure, random_tree, words_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
KINDS = pytest.mark.parametrize("code", [None, 0, 1], ids=["pools", "int8", "e4m3"])
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    yield ts
    torch.cuda.empty_cache()


def dev(x):
    from paper_2411_02886_amd.runtime import to_device
    return to_device(x)


class Held:
    """What a sequence's tokens hold, in 64 bits, as tree_util.attention reads it."""

    def __init__(self, dtype, k, v, lens):
        self.dtype, self.H_kv, self.lens = dtype, k[0].shape[1], np.asarray(lens, np.int32)
        self.start = np.cumsum([0] + [int(n) for n in lens])
        self.k, self.v = np.concatenate(k), np.concatenate(v)

    def slots(self, b):
        return np.arange(self.start[b], self.start[b + 1])


@DTYPES
@KINDS
@pytest.mark.parametrize("H,H_kv,D,n", [(8, 2, 64, 9), (28, 4, 128, 40)])
def test_drafts_are_attended_kept_and_gone_on_from(gpu, dtype, code, H, H_kv, D, n):
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import DecodeLayer, copy_pages, to_host
    P, NP = 16, 64
    rng = np.random.default_rng(n)
    sdt = torch.int16 if dtype == BF else torch.float32
    k_pool, v_pool = (torch.zeros((NP, P, H_kv, D), dtype=sdt, device="cuda:0") for _ in "kv")
    cache = None if code is None else gpu.QuantCache.empty(NP, P, H_kv, D, code)
    pool, sm = PagePool(NP, P), 1 / math.sqrt(D)
    rope = gpu.Rope(inv_freq=dev((1e4 ** -(np.arange(16) / 16)).astype(np.float32)))

    def rows(m, h):
        return W.store(rng.standard_normal((m, h, D), dtype=np.float32), dtype)

    def layer(seqs):
        ind, pages, lens = pool.table(seqs)
        return DecodeLayer(dtype=dtype, H=H, H_kv=H_kv, D=D, P=P, k=8, k_pool=k_pool, v_pool=v_pool, page_indptr=ind, page_indices=pages,
                           seq_lens=lens, max_seq_len=400)

    def held(lay, seqs):
        """The tokens as they stand in the pages."""
        lens = lay.seq_lens.cpu().numpy()
        if cache is not None:
            T = int(lens.sum())
            out = [torch.full((T, H_kv, D), 7, dtype=sdt, device="cuda:0") for _ in "kv"]
            lay.read_back(cache, *out, q_indptr=dev(np.cumsum([0] + lens.tolist()).astype(np.int32)))
            torch.cuda.synchronize()
            kc, vc, ks, vs = (to_host(t) for t in cache._keep)
            exact = [of_code(x.reshape(-1, H_kv, D), code) * y.transpose(0, 2, 1).reshape(-1, H_kv)[..., None].astype(np.float64) for x, y in ((kc, ks), (vc, vs))]
        else:
            exact = [W.as_f32(to_host(t, bits16=dtype == BF), dtype).astype(np.float64).reshape(-1, H_kv, D) for t in (k_pool, v_pool)]
        slot = [np.array(pool.pages(s))[np.arange(m) // P] * P + np.arange(m) % P for s, m in zip(seqs, lens)]
        k, v = ([x[at] for at in slot] for x in exact)
        if cache is not None:                            # a code times its scale, rounded to float and to the type
            for got, want in zip(out, (k, v)):
                want = np.concatenate(want)
                got = W.as_f32(to_host(got, bits16=dtype == BF), dtype)
                assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -24 if dtype == BF else 2.0 ** -24) * np.abs(want))
        return Held(dtype, k, v, lens)

    def attend(lay, seqs, q, new, mask=None, sees=None, most=None):
        T = sum(new)
        ind = dev(np.cumsum([0] + new).astype(np.int32))
        out, lse = torch.zeros((T, H, D), dtype=sdt, device="cuda:0"), torch.zeros((T, H), device="cuda:0")
        lay.attend_all(q, q_indptr=ind, out=out, lse=lse, most_new=most, mask=mask, cache=cache)
        torch.cuda.synchronize()
        ref = attention(held(lay, seqs), to_host(q, bits16=dtype == BF), new, 0, float(np.float32(sm)), sees, more=4, tiny=2.0 ** -108)
        check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64), ref, new)

    def append(lay, new, positions=None):
        T = sum(new)
        q, k, v = rows(T, H), rows(T, H_kv), rows(T, H_kv)
        q_out = torch.zeros((T, H, D), dtype=sdt, device="cuda:0")
        lay.append(dev(k), dev(v), q=dev(q), q_out=q_out, rope=rope, positions=positions, q_indptr=dev(np.cumsum([0] + new).astype(np.int32)), cache=cache)
        return q_out, k, v

    def copies_of(lay, copies):
        copy_pages(lay.problem, copies, NP, cache=cache)

    # prompts of a and b, then c goes on from b in pages of its own
    for s, m in (("a", 37), ("b", 90)):
        pool.add(s)
        pool.grow(s, m)
        lay = layer([s])
        attend(lay, [s], append(lay, [m])[0], [m], most=m)
    pool.fork("b", "c")
    seqs = ["a", "b", "c"]

    for step in range(3):
        # a tree for each, of different sizes; c writes behind pages that it shares with b until it gets its own
        new = [n, max(1, n - 5 * step), n + step]
        old = [pool.length(s) for s in seqs]
        for s, m in zip(seqs, new):
            copies_of(layer([s]), pool.grow(s, m))
        lay = layer(seqs)
        before = held(lay, seqs)
        T, words = sum(new), (max(new) + 31) // 32
        parents = [random_tree(rng, m, roots=step == 1) for m in new]
        ind = dev(np.cumsum([0] + new).astype(np.int32))
        mask, pos = torch.zeros((T, words), dtype=torch.int32, device="cuda:0"), torch.zeros((1, T), dtype=torch.int32, device="cuda:0")
        lay.tree_mask(dev(np.concatenate(parents)), mask, positions=pos, q_indptr=ind)
        sees = [closure(x) for x in parents]
        q, k, v = append(lay, new, positions=pos)
        attend(lay, seqs, q, new, mask=mask, sees=sees, most=max(new))
        now = held(lay, seqs)
        for b in range(3):                               # what was there stays
            at = now.slots(b)[:old[b]]
            assert np.array_equal(now.k[at], before.k[at]) and np.array_equal(now.v[at], before.v[at])
        # accept a path of each: a node that nobody follows, and all that lead to it; of b nothing in the second step
        paths = [np.flatnonzero(sees[b][int(rng.integers(0, new[b]))]) for b in range(3)]
        if step == 1:
            paths[1] = paths[1][:0]
        stride = max(len(x) for x in paths)
        path = np.full((3, stride), -1, np.int32)
        for b, x in enumerate(paths):
            path[b, :len(x)] = x
        to_lens = torch.zeros(3, dtype=torch.int32, device="cuda:0")
        lay.keep(dev(path), dev(np.array([len(x) for x in paths], np.int32)), to_lens, q_indptr=ind, cache=cache)
        lay.seq_lens.copy_(to_lens)
        torch.cuda.synchronize()
        lens = [o + len(x) for o, x in zip(old, paths)]
        assert to_lens.cpu().tolist() == lens
        kept = held(lay, seqs)
        for b in range(3):
            was = now.slots(b)
            want = np.concatenate([was[:old[b]], was[old[b] + paths[b]]])
            assert np.array_equal(kept.k[kept.slots(b)], now.k[want]) and np.array_equal(kept.v[kept.slots(b)], now.v[want])
        # V of the path is what was appended
        for b, x in enumerate(paths):
            mine = v[sum(new[:b]) + x]
            stored = W.as_f32(mine, dtype).astype(np.float64)
            if cache is not None:
                codes, scales = encode(stored, code)
                stored = of_code(codes, code) * scales[..., None].astype(np.float64)
            assert np.array_equal(kept.v[kept.slots(b)[old[b]:]], stored)
        for s, m in zip(seqs, lens):
            pool.cut(s, m)
        # the model's own next token behind it
        for s in seqs:
            copies_of(layer([s]), pool.grow(s))
        lay = layer(seqs)
        attend(lay, seqs, append(lay, [1] * 3)[0], [1] * 3)



@DTYPES
@KINDS
def test_a_captured_step_of_drafts_gives_what_the_calls_give(gpu, dtype, code):
    """Mask, append, attention and keep in one graph, replayed with other trees, lengths and paths."""
    from paper_2411_02886_amd.runtime import DecodeLayer
    B, n, H, H_kv, D, P, NP = 3, 12, 8, 2, 64, 16, 200
    rng = np.random.default_rng(5)
    sdt = torch.int16 if dtype == BF else torch.float32
    room = 60
    pages = rng.permutation(NP)[:B * room].astype(np.int32)
    k_pool, v_pool = (dev(W.store(rng.standard_normal((NP, P, H_kv, D), dtype=np.float32), dtype)) for _ in "kv")
    cache = None if code is None else gpu.QuantCache.empty(NP, P, H_kv, D, code)
    lay = DecodeLayer(dtype=dtype, H=H, H_kv=H_kv, D=D, P=P, k=8, k_pool=k_pool, v_pool=v_pool, page_indptr=np.arange(B + 1) * room, page_indices=pages,
                      seq_lens=np.array([900, 30, 500]), max_seq_len=room * P)
    rope = gpu.Rope(inv_freq=dev((1e4 ** -(np.arange(16) / 16)).astype(np.float32)))
    if cache is not None:                                # fill it
        at = dev(np.array([0, 888, 906, 1394], np.int32))
        lay.seq_lens.copy_(dev(np.array([888, 18, 488], np.int32)))
        lay.append(*(dev(W.store(rng.standard_normal((1394, H_kv, D), dtype=np.float32), dtype)) for _ in "kv"), rope=rope, q_indptr=at, cache=cache)
    ind, T = dev(np.arange(B + 1, dtype=np.int32) * n), B * n
    q, k, v = (dev(W.store(rng.standard_normal((T, h, D), dtype=np.float32), dtype)) for h in (H, H_kv, H_kv))
    parents, path, count = torch.zeros(T, dtype=torch.int32, device="cuda:0"), torch.zeros((B, n), dtype=torch.int32, device="cuda:0"), torch.zeros(B, dtype=torch.int32, device="cuda:0")
    mask, pos, to_lens = (torch.zeros(x, dtype=torch.int32, device="cuda:0") for x in ((T, 1), (1, T), (B,)))
    q_out, out, lse = torch.zeros((T, H, D), dtype=sdt, device="cuda:0"), torch.zeros((T, H, D), dtype=sdt, device="cuda:0"), torch.zeros((T, H), device="cuda:0")
    ws = torch.empty(1 << 23, dtype=torch.int32, device="cuda:0")

    def step():
        lay.tree_mask(parents, mask, positions=pos, q_indptr=ind)
        lay.append(k, v, q=q, q_out=q_out, rope=rope, positions=pos, q_indptr=ind, cache=cache)
        lay.attend_all(q_out, q_indptr=ind, out=out, lse=lse, most_new=n, mask=mask, cache=cache, ws=ws)
        lay.keep(path, count, to_lens, q_indptr=ind, cache=cache)

    def draw(lens):
        trees = [random_tree(rng, n) for _ in range(B)]
        parents.copy_(torch.from_numpy(np.concatenate(trees)))
        lay.seq_lens.copy_(torch.from_numpy(np.array(lens, np.int32)))
        rows = np.zeros((B, n), np.int32)
        counts = []
        for b in range(B):
            x = np.flatnonzero(closure(trees[b])[n - 1 - b])
            rows[b, :len(x)] = x
            counts.append(len(x))
        path.copy_(torch.from_numpy(rows))
        count.copy_(torch.from_numpy(np.array(counts, np.int32)))

    state = [k_pool, v_pool] if cache is None else list(cache._keep)
    results = [mask, pos, q_out, out, lse, to_lens]
    draw([900, 30, 500])
    stream = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(stream):
        step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        step()
    for lens in ([900, 30, 500], [13, 12, 700], [960, 200, 5]):
        draw(lens)
        began = [x.clone() for x in state]
        for x in results:
            x.zero_()
        step()
        torch.cuda.synchronize()
        want = [x.clone() for x in results + state]
        for x, y in zip(state, began):
            x.copy_(y)
        for x in results:
            x.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for x, y in zip(results + state, want):
            assert torch.equal(x, y), lens


POOL_BYTES = 5 << 30


@pytest.mark.parametrize("dtype,code,H,H_kv,D,P,lens", [(BF, 0, 32, 8, 128, 16, [6000, 3333, 70]), (F32, 1, 8, 2, 64, 8, [2500, 700, 33]),
                                                        (BF, 1, 16, 16, 64, 64, [1800, 900, 64])], ids=["bf16", "f32", "mha"])
def test_a_cache_beyond_4_gib(gpu, dtype, code, H, H_kv, D, P, lens):
    """Codes of 5 GiB for K and V each, the pages in use scattered over them, three quarters above the 4 GiB line and one at the very end."""
    rng = np.random.default_rng(P)
    c = QuantPages(dtype, code, H_kv, D, P, lens, seed=P, spare=40 // P + 1)
    page_bytes = P * H_kv * D
    NP, line, m = POOL_BYTES // page_bytes, (4 << 30) // page_bytes, c.num_pages
    below = rng.choice(line, size=m // 4, replace=False)
    above = line + rng.choice(NP - 1 - line, size=m - m // 4 - 1, replace=False)
    ids = np.concatenate([below, above, [NP - 1]])
    rng.shuffle(ids)
    last, other = c.pages[-1], int(np.flatnonzero(ids == NP - 1)[0])
    ids[[last, other]] = ids[[other, last]]              # the end belongs to the last sequence
    cache = gpu.QuantCache.empty(NP, P, H_kv, D, code)
    at = torch.from_numpy(ids).to("cuda:0")
    _, small = c.problem(H)
    for big, x in zip(cache._keep, small._keep):
        big[at] = x.view(big.dtype)
    z, sm = dev(c.indptr), float(np.float32(1 / math.sqrt(D)))

    def problem(chunk=1, most=None):
        return gpu.Problem(batch=3, chunk=chunk, num_q_heads=H, num_kv_heads=H_kv, head_dim=D, page_size=P, max_seq_len=most or max(lens), dtype=dtype, k_pool=None, v_pool=None,
                           page_indptr=z, page_indices=dev(ids[c.pages].astype(np.int32)), seq_lens=dev(c.lens))

    from paper_2411_02886_amd.runtime import to_host
    sdt = torch.int16 if dtype == BF else torch.float32
    for new, most in (([1] * 3, None), ([1] * 3, 1 << 24), ([40, 33, 30], None)):
        T, sees = sum(new), None if new[0] == 1 else [closure(random_tree(rng, x)) for x in new]
        p = problem(max(new), most)
        q = W.store(rng.standard_normal((T, H, D), dtype=np.float32), dtype)
        out, lse = torch.zeros((T, H, D), dtype=sdt, device="cuda:0"), torch.zeros((T, H), device="cuda:0")
        ws = torch.empty(gpu.ts_quant_attn_workspace_bytes(p, T) // 4, dtype=torch.int32, device="cuda:0")
        mask = None if sees is None else dev(np.concatenate([words_of(x, 2) for x in sees]).view(np.int32))
        gpu.ts_quant_attn(p, cache, dev(q), dev(np.cumsum([0] + new).astype(np.int32)), T, 0, mask, sm, out, lse, ws)
        torch.cuda.synchronize()
        check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64),
                        attention(c, q, new, 0, sm, sees, more=4, tiny=2.0 ** -108), (new, most))
    # new rows are written where the pages are, read back, and moved within them
    new = [20, 33, 30]
    T, ind = sum(new), dev(np.cumsum([0] + [20, 33, 30]).astype(np.int32))
    k, v = (W.store(rng.standard_normal((T, H_kv, D), dtype=np.float32), dtype) for _ in "kv")
    p = problem(max(new))
    gpu.ts_quant_append(p, cache, None, None, dev(k), dev(v), ind, T, None, None)
    path, count, to_lens = np.array([[1, 5, 19], [0, 30, 32], [2, 3, 29]], np.int32), dev(np.array([3, 2, 3], np.int32)), torch.zeros(3, dtype=torch.int32, device="cuda:0")
    gpu.ts_tree_keep(p, cache, dev(path), 3, count, ind, to_lens)
    back = [torch.zeros((T, H_kv, D), dtype=sdt, device="cuda:0") for _ in "kv"]
    gpu.ts_quant_read(p, cache, ind, T, *back)
    src, dst = int(ids[c.pages[-1]]), int(ids[c.spare[0]])
    gpu.ts_quant_pages_copy(p, cache, dev(np.array([src], np.int32)), dev(np.array([dst], np.int32)), 1, NP)
    torch.cuda.synchronize()
    assert src == NP - 1
    for name, rows, codes, scale, got in zip("kv", (k, v), cache._keep[:2], cache._keep[2:], back):
        want_c, want_s = c.bytes[name].copy(), c.scales[name].copy()
        cc, ss = encode(W.as_f32(rows, dtype).astype(np.float64), code)
        first = 0
        for b, m in enumerate(new):
            slots = c.slots(b)[lens[b] - m:]
            want_c[slots], want_s[slots] = cc[first:first + m], ss[first:first + m]
            take = path[b, :3 if b != 1 else 2]
            moved = want_c[slots[take]].copy(), want_s[slots[take]].copy()
            want_c[slots[:len(take)]], want_s[slots[:len(take)]] = moved
            first += m
        used = np.unique(c.pages)
        got_c = to_host(codes[at]).reshape(-1, P, H_kv, D)
        got_s = to_host(scale[at]).transpose(0, 2, 1)
        assert np.array_equal(got_c[used], want_c.reshape(-1, P, H_kv, D)[used])
        assert np.array_equal(got_s[used], want_s.reshape(-1, P, H_kv)[used], equal_nan=True)
        assert np.array_equal(got_c[c.spare[0]], got_c[c.pages[-1]]) and np.array_equal(got_s[c.spare[0]], got_s[c.pages[-1]], equal_nan=True)
        values = c.values(want_c, want_s)
        want = np.concatenate([values[c.slots(b)[lens[b] - m:]] for b, m in enumerate(new)])
        got = W.as_f32(to_host(got, bits16=dtype == BF), dtype)
        assert np.all(np.abs(got - want) <= (2.0 ** -8 + 2.0 ** -24 if dtype == BF else 2.0 ** -24) * np.abs(want))
    # nothing else of the codes was touched
    for codes in cache._keep[:2]:
        rest = torch.ones(NP, dtype=torch.bool, device="cuda:0")
        rest[at] = False
        assert not any(bool((codes[a:a + (NP >> 4)][rest[a:a + (NP >> 4)]] != 0).any()) for a in range(0, NP, NP >> 4))
