"""ts_pages_copy and ts_cache_compact: every byte of the pools afterwards, and the calls together as a server uses them."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache

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


def bits(t):
    a = t.cpu().numpy()
    return a.view(np.uint16 if a.dtype == np.int16 else np.uint32)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H_kv,D,P", [(1, 64, 8), (2, 64, 16), (8, 128, 1), (8, 128, 16), (32, 128, 64), (4, 128, 256)])
@pytest.mark.parametrize("with_v", [True, False], ids=["kv", "k"])
def test_pages_copy(gpu, dtype, H_kv, D, P, with_v):
    from paper_2411_02886_amd.runtime import to_device
    rng = np.random.Generator(np.random.PCG64(P))
    n, pages = 17, 50
    dt = torch.int16 if dtype == BF else torch.int32
    k, v = (torch.randint(-30000, 30000, (pages, P, H_kv, D), dtype=dt, device="cuda:0") for _ in "kv")
    k0, v0 = k.clone(), v.clone()
    perm = rng.permutation(pages)
    src, dst = perm[:n].astype(np.int32), perm[n:2 * n].astype(np.int32)
    src[3] = src[5]                                       # one page may go to several places
    src[7], dst[8], src[9], dst[10] = -1, -1, pages, pages + 7   # skipped
    src[11] = dst[11]                                     # onto itself
    z = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    p = gpu.Problem(batch=1, num_q_heads=H_kv, num_kv_heads=H_kv, head_dim=D, page_size=P, max_seq_len=1, dtype=dtype, k_pool=k,
                    v_pool=v if with_v else None, page_indptr=z, page_indices=z, seq_lens=z)
    gpu.ts_pages_copy(p, to_device(src), to_device(dst), n, pages)
    torch.cuda.synchronize()
    for s, d in zip(src, dst):
        if 0 <= s < pages and 0 <= d < pages:
            k0[d] = k[s] if s == d else k0[s]
            if with_v:
                v0[d] = v0[s]
    assert torch.equal(k, k0) and torch.equal(v, v0)
    gpu.ts_pages_copy(p, None, None, 0, pages)            # nothing to do


def test_more_pairs_than_a_grid_holds(gpu):
    n = 40000
    k = torch.arange(2 * n, dtype=torch.int32, device="cuda:0")[:, None].repeat(1, 64).view(2 * n, 1, 1, 64)
    src, dst = torch.arange(n, dtype=torch.int32, device="cuda:0"), torch.arange(n, 2 * n, dtype=torch.int32, device="cuda:0")
    z = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    p = gpu.Problem(batch=1, num_q_heads=1, num_kv_heads=1, head_dim=64, page_size=1, max_seq_len=1, dtype=F32, k_pool=k, v_pool=None,
                    page_indptr=z, page_indices=z, seq_lens=z)
    gpu.ts_pages_copy(p, src, dst, n, 2 * n)
    torch.cuda.synchronize()
    assert torch.equal(k[n:], k[:n])


def compacted(c, idx, count, n_init, n_local, to_indptr, to_pages, skip):
    """Pools and lengths after the call, by the definition, and the kept tokens."""
    k, v, lens, kept = c.k_bits.copy(), c.v_bits.copy(), [], []
    for b in range(c.B):
        n = int(c.lens[b])
        lo = min(n_init, n)
        hi = max(lo, n - n_local)
        m = min(max(int(count[b]), 0), idx.shape[1]) if n else 0
        t = np.concatenate([np.arange(lo), np.clip(idx[b, :m], 0, max(n - 1, 0)), np.arange(hi, n)]).astype(int)
        t = t[:max(0, int(to_indptr[b + 1] - to_indptr[b])) * c.P]
        kept.append(t)
        lens.append(-7 if skip is not None and skip[b] else len(t))
        if skip is not None and skip[b]:
            continue
        j = np.arange(len(t))
        at = to_pages[to_indptr[b] + j // c.P].astype(np.int64) * c.P + j % c.P
        k[at], v[at] = c.k_bits[c.slots(b)[t]], c.v_bits[c.slots(b)[t]]
    return k, v, lens, kept


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H_kv,D,P,n_init,n_local", [(2, 64, 16, 0, 0), (1, 64, 8, 4, 9), (8, 128, 16, 128, 33), (32, 128, 1, 3, 0), (4, 128, 64, 0, 70)])
@pytest.mark.parametrize("odd", [False, True], ids=["", "odd"])
def test_cache_compact(gpu, dtype, H_kv, D, P, n_init, n_local, odd):
    from paper_2411_02886_amd.runtime import to_device
    rng = np.random.Generator(np.random.PCG64(P + n_init))
    lens, k = [300, 0, 1, 77, 1000], 90
    c = Cache(dtype, H_kv, D, P, lens, seed=P, spare=5 * (-(-(k + n_init + n_local) // P)))
    idx, count = np.full((5, k), -1, np.int32), np.zeros(5, np.int32)
    for b, n in enumerate(lens):
        lo = min(n_init, n)
        hi = max(lo, n - n_local)
        m = min(k, hi - lo)
        idx[b, :m] = np.sort(lo + rng.permutation(hi - lo)[:m])
        count[b] = m
    skip, to = None, [(-(-(k + n_init + n_local) // P))] * 5
    if odd:         # a skipped sequence, corrupt lists, too few pages, a count for a sequence without tokens
        skip = np.array([0, 0, 0, 1, 0], np.uint8)
        idx[0, 3], idx[0, 4], count[1], count[4] = -5, 1 << 30, 9, k + 50
        to[4] = max(0, to[4] - 1)
        to[2] = 0
    to_indptr = np.cumsum([0] + to).astype(np.int32)
    want = compacted(c, idx, count, n_init, n_local, to_indptr, c.spare, skip)
    p, kp, vp = c.problem(H_kv, num_initial=n_init, num_local=n_local)
    new = torch.full((5,), -7, dtype=torch.int32, device="cuda:0")
    gpu.ts_cache_compact(p, to_device(idx), k, to_device(count), None if skip is None else to_device(skip), to_device(to_indptr),
                         to_device(c.spare), new)
    torch.cuda.synchronize()
    assert new.cpu().tolist() == want[2]
    for t, w in zip((kp, vp), want):
        assert np.array_equal(bits(t).reshape(-1), np.ascontiguousarray(w).reshape(-1).view(np.uint16 if dtype == BF else np.uint32))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_append_attend_select_compact_and_attend_again(gpu, dtype):
    """A server's turn: prompts are appended and attended, a child forks and both go on in pages of their own, the selection attends, the cache
    is cut down to it and attending all of what is left gives what the selection gave."""
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import ChunkSelector, DecodeLayer, copy_pages, to_device
    H, H_kv, D, P, C, k = 8, 2, 64, 16, 45, 48
    rng = np.random.default_rng(3)
    tdt, sdt = (torch.bfloat16, torch.int16) if dtype == BF else (torch.float32, torch.float32)
    NP = 120
    k_pool, v_pool = (torch.full((NP, P, H_kv, D), 0, dtype=sdt, device="cuda:0") for _ in "kv")
    pool = PagePool(NP, P)
    rope = gpu.Rope(inv_freq=to_device((1e4 ** -(np.arange(32) / 32)).astype(np.float32)))

    def rows(n, h):
        return to_device(W.store(rng.standard_normal((n, h, D), dtype=np.float32), dtype))

    def layer(seqs, **kw):
        ind, pages, lens = pool.table(seqs)
        return DecodeLayer(dtype=dtype, H=H, H_kv=H_kv, D=D, P=P, k=k, k_pool=k_pool, v_pool=v_pool, page_indptr=ind,
                           page_indices=pages, seq_lens=lens, **kw)

    def full(seq, q):
        """The turned query's attention over the whole sequence in 64 bits, from the pools' contents."""
        n = pool.length(seq)
        t = np.arange(n)
        slot = torch.tensor(np.array(pool.pages(seq))[t // P] * P + t % P, device="cuda:0")
        kk, vv = (x.view(tdt).view(-1, H_kv, D)[slot].double().cpu() for x in (k_pool, v_pool))
        z = torch.einsum("hgd,nhd->hgn", q.view(tdt).double().cpu().view(H_kv, H // H_kv, D), kk) / math.sqrt(D)
        return torch.einsum("hgn,nhd->hgd", torch.softmax(z, -1), vv).reshape(H, D)

    # two prompts of 45 and 90 tokens, in chunks of 45, attended as they come
    for s, chunks in (("a", 1), ("b", 2)):
        pool.add(s)
        for _ in range(chunks):
            copy_pages(None, pool.grow(s, C), NP)
            if dtype == BF:
                ind, pages, lens = pool.table([s])
                sel = ChunkSelector(C=C, H=H, H_kv=H_kv, D=D, P=P, k=k, k_pool=k_pool, v_pool=v_pool, page_indptr=ind,
                                    page_indices=pages, seq_lens=lens)
                q, q_out = rows(C, H), torch.empty((C, H, D), dtype=sdt, device="cuda:0")
                sel.append(rows(C, H_kv), rows(C, H_kv), q=q, q_out=q_out, rope=rope)
                sel.attend_all(q_out)
                torch.cuda.synchronize()
                got = sel.out[0, -1].view(tdt).double().cpu()
            else:       # the chunk selection is bf16 only; its layer's calls on packed rows serve both
                lay = layer([s])
                q, q_out = rows(C, H), torch.empty((C, H, D), dtype=sdt, device="cuda:0")
                ind = to_device(np.array([0, C], np.int32))
                lay.append(rows(C, H_kv), rows(C, H_kv), q=q, q_out=q_out, rope=rope, q_indptr=ind)
                out = torch.empty((C, H, D), dtype=sdt, device="cuda:0")
                lay.attend_all(q_out, q_indptr=ind, out=out)
                torch.cuda.synchronize()
                got = out[-1].double().cpu()
            want = full(s, q_out[-1])
            # weights and result rounded to bf16: two half steps of sums of |v| weights (|v| < 5 here); float: far below 1e-5
            assert (got - want).abs().max() <= (2 * 2.0 ** -8 * 5 if dtype == BF else 1e-5)

    # a child of b; both append one token: the child's write must not reach the parent's page
    pool.fork("b", "c")
    assert pool.pages("b") == pool.pages("c")
    lay = layer(["b"])
    for s in ("c", "b"):
        copy_pages(lay.problem, pool.grow(s), NP)
    assert pool.pages("b")[:-1] == pool.pages("c")[:-1] and pool.pages("b")[-1] != pool.pages("c")[-1]
    lay = layer(["a", "b", "c"], max_seq_len=200)
    copies = pool.grow("a")
    assert not copies
    lay = layer(["a", "b", "c"], max_seq_len=200, num_initial=4, num_local=8)
    q, q_out = rows(3, H), torch.empty((3, H, D), dtype=sdt, device="cuda:0")
    lay.append(rows(3, H_kv), rows(3, H_kv), q=q, q_out=q_out, rope=rope)
    lay.attend_all(q_out)
    torch.cuda.synchronize()
    for i, s in enumerate("abc"):
        want = full(s, q_out[i])
        assert (lay.out[i, 0].view(tdt).double().cpu() - want).abs().max() <= (2.0 ** -8 * 5 if dtype == BF else 1e-5), s

    # selection, and the cache cut down to it
    lay.step(q_out.view(3, 1, H, D))
    sparse, sparse_lse = lay.out.clone(), lay.lse.clone()
    spare = [pool.spare(4 + k + 8) for _ in range(3)]
    to_indptr, to_pages = np.cumsum([0] + [len(x) for x in spare]).astype(np.int32), np.concatenate(spare).astype(np.int32)
    to_lens = torch.zeros(3, dtype=torch.int32, device="cuda:0")
    lay.compact(to_device(to_indptr), to_device(to_pages), to_lens)
    lens = to_lens.cpu().tolist()
    assert lens == [46, 60, 60]
    for s, pages, n in zip("abc", spare, lens):
        pool.replace(s, pages, n)
    assert pool.free_pages == NP - sum(-(-n // P) for n in lens)
    # the pages move to the low end of the pool, and attending all of them is what the selection attended
    moves = pool.gather()
    assert moves and max(max(pool.pages(s)) for s in "abc") < 11
    copy_pages(lay.problem, moves, NP)
    small = layer(["a", "b", "c"])
    small.attend_all(q_out)
    torch.cuda.synchronize()
    # the same sums in another order: a rounding of the type between them (bf16: a step of values below 5), and the float sums' own error
    tol = 2.0 ** -8 * 5 * 2 if dtype == BF else 1e-5
    assert (small.out.view(tdt).double() - sparse.view(tdt).double()).abs().max() <= tol
    assert (small.lse - sparse_lse).abs().max() <= 1e-5
    for s in "abc":
        pool.free(s)
    assert pool.free_pages == NP and not pool.refs.any()


def test_captured_copies_and_compactions_read_their_lists_when_they_run(gpu):
    from paper_2411_02886_amd.runtime import to_device
    c = Cache(BF, 2, 64, 16, [60, 33], seed=2, spare=12)
    p, kp, vp = c.problem(2, num_initial=2, num_local=3)
    src, dst = to_device(c.pages[:3].copy()), to_device(c.spare[:3].copy())
    idx = to_device(np.array([[5, 9, 20, 44], [3, 4, 5, 6]], np.int32))
    count, new = to_device(np.array([4, 2], np.int32)), torch.zeros(2, dtype=torch.int32, device="cuda:0")
    to_indptr, to = to_device(np.array([0, 2, 4], np.int32)), to_device(c.spare[4:8].copy())
    k0, v0 = kp.clone(), vp.clone()

    def call():
        gpu.ts_pages_copy(p, src, dst, 3, kp.shape[0])
        gpu.ts_cache_compact(p, idx, 4, count, None, to_indptr, to, new)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for rep in range(4):
        kp.copy_(k0); vp.copy_(v0); new.zero_(); torch.cuda.synchronize()
        g.replay(); torch.cuda.synchronize()
        got = [t.clone() for t in (kp, vp, new)]
        kp.copy_(k0); vp.copy_(v0); new.zero_()
        call(); torch.cuda.synchronize()
        for a, b in zip(got, (kp, vp, new)):
            assert torch.equal(a, b), rep
        idx += 1
        dst.copy_(dst.roll(1))
