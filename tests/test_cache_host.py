"""What the cache's calls refuse (nothing is launched), and the page table on the host."""
import ctypes

import numpy as np
import pytest

import paper_2411_02886_amd as ts
from paper_2411_02886_amd.binding import _CProblem, _CRope
from paper_2411_02886_amd.pages import PagePool

torch = pytest.importorskip("torch")
A, BIG = 0x10000, 1 << 40
OK, BAD, UNSUP, WS = 0, -1, -2, -3


def cproblem(**kw):
    base = dict(batch=2, chunk=1, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=4096, dtype=ts.TS_BF16,
                k_pool=A, v_pool=A, page_indptr=A, page_indices=A, seq_lens=A, num_initial=0, num_local=0)
    base.update(kw)
    return _CProblem(**base)


def attn(p=None, q=A, ind=None, rows=2, window=0, sm=0.1, out=0x900000, lse=None, ws=0x2000000, ws_bytes=BIG):
    return ts.load().ts_paged_attn(ctypes.byref(p or cproblem()), q, ind, rows, window, sm, out, lse, ws, ws_bytes, None)


def test_paged_attn_refusals():
    for kw in (dict(q=None), dict(out=None), dict(rows=3), dict(rows=-1), dict(window=-1), dict(sm=float("nan")), dict(sm=float("inf")),
               dict(q=A + 8), dict(out=0x900004), dict(out=A), dict(out=A + 2 * 8 * 64 * 2 - 16),
               dict(p=cproblem(v_pool=None)), dict(p=cproblem(k_pool=None)), dict(p=cproblem(k_pool=A + 2)), dict(p=cproblem(seq_lens=None)),
               dict(p=cproblem(num_q_heads=7))):
        assert attn(**kw) == BAD, kw
    assert attn(p=cproblem(head_dim=96)) == UNSUP and attn(p=cproblem(page_size=12)) == UNSUP
    for kw in (dict(ws=None), dict(ws=0x2000010), dict(ws_bytes=16)):
        assert attn(**kw) == WS, kw
    assert attn(rows=0, q=None, out=None, ws=None, ws_bytes=0) == OK
    assert attn(ind=A, rows=0) == OK


def test_paged_attn_workspace():
    L, out = ts.load(), ctypes.c_size_t(0)
    get = lambda rows, **kw: (L.ts_paged_attn_workspace_bytes(ctypes.byref(cproblem(**kw)), rows, ctypes.byref(out)), out.value)
    assert get(-1)[0] == BAD and L.ts_paged_attn_workspace_bytes(None, 1, ctypes.byref(out)) == BAD
    assert get(1, head_dim=80)[0] == UNSUP
    # one workspace serves every call with fewer rows, shorter chunks and sequences, fewer sequences
    for dtype in (ts.TS_BF16, ts.TS_F32):
        for H, H_kv, D in ((8, 2, 64), (32, 8, 128), (28, 4, 128), (3, 1, 64), (128, 32, 128)):
            shape = dict(num_q_heads=H, num_kv_heads=H_kv, head_dim=D, dtype=dtype)
            for axis, values in (("rows", [0, 1, 2, 31, 33, 64, 500, 5000, 100000]), ("chunk", [1, 2, 3, 4, 8, 9, 16, 17, 64, 500, 9000]),
                                 ("batch", [1, 2, 7, 64, 300, 5000]), ("max_seq_len", [1, 100, 1000, 5000, 100000, 1 << 20])):
                last = 0
                for x in values:
                    rows, kw = 64, dict(chunk=20, batch=3, max_seq_len=20000)
                    if axis == "rows":
                        rows = x
                    else:
                        kw[axis] = x
                    st, n = get(rows, **kw, **shape)
                    assert st == OK and n >= last and n % 256 == 0, (axis, x)
                    last = n


def rope(**kw):
    base = dict(inv_freq=A, rotary_dim=64, num_axes=1, adjacent=0, scale=1.0)
    axes = kw.pop("pair_axis", [0] * 64)
    base.update(kw)
    return _CRope(**base, pair_axis=(ctypes.c_uint8 * 64)(*axes))


def append(p=None, r=None, q=A, qs=0, k=0x200000, ks=0, v=0x300000, vs=0, ind=None, rows=2, pos=None, out=0x900000):
    return ts.load().ts_rope_append(ctypes.byref(p or cproblem()), ctypes.byref(r) if r is not None else None, q, qs, k, ks, v, vs, ind, rows,
                                    pos, out, None)


def test_rope_append_refusals():
    for r in (dict(rotary_dim=63), dict(rotary_dim=66), dict(rotary_dim=-2), dict(num_axes=0), dict(num_axes=5), dict(adjacent=2),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(inv_freq=None), dict(pair_axis=[0] * 31 + [1] + [0] * 32)):
        assert append(r=rope(**r)) == BAD, r
    for kw in (dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(q=None, out=None, k=None, v=None), dict(rows=3), dict(rows=-2),
               dict(q=A + 4), dict(out=0x900002), dict(k=0x200008), dict(v=0x300001), dict(qs=500), dict(qs=516), dict(ks=100), dict(ks=132),
               dict(vs=-128), dict(p=cproblem(k_pool=None)), dict(p=cproblem(v_pool=None)), dict(p=cproblem(k_pool=A + 8)),
               dict(out=A + 1024), dict(q=A, out=A, qs=1024), dict(out=0x200000), dict(out=0x300000 - 64)):
        assert append(r=rope(), **kw) == BAD, kw
    assert append(p=cproblem(head_dim=32)) == UNSUP
    assert append(rows=0, q=None, out=None, k=None, v=None) == OK
    # a part of a pair table that no pair reaches does not count
    assert append(r=rope(rotary_dim=2, pair_axis=[0] + [9] * 63), rows=0) == OK
    assert append(r=rope(rotary_dim=4, pair_axis=[0] + [9] * 63), rows=0) == BAD


def test_pages_copy_and_compact_refusals():
    L = ts.load()
    copy = lambda p=None, src=A, dst=A, n=2, pages=9: L.ts_pages_copy(ctypes.byref(p or cproblem()), src, dst, n, pages, None)
    for kw in (dict(src=None), dict(dst=None), dict(n=-1), dict(pages=0), dict(p=cproblem(k_pool=None)), dict(p=cproblem(k_pool=A + 8)),
               dict(p=cproblem(v_pool=A + 4))):
        assert copy(**kw) == BAD, kw
    assert copy(n=0, src=None, dst=None) == OK and copy(p=cproblem(num_kv_heads=3, num_q_heads=3)) == UNSUP
    compact = lambda p=None, idx=A, stride=4, count=A, skip=None, ti=A, tp=A, tl=A: L.ts_cache_compact(
        ctypes.byref(p or cproblem()), idx, stride, count, skip, ti, tp, tl, None)
    for kw in (dict(idx=None), dict(stride=0), dict(count=None), dict(ti=None), dict(tp=None), dict(tl=None), dict(p=cproblem(v_pool=None)),
               dict(p=cproblem(v_pool=A + 8))):
        assert compact(**kw) == BAD, kw
    assert compact(p=cproblem(chunk=2)) == UNSUP


def test_binding_refuses_what_the_library_cannot_see():
    f = torch.ones(32)
    assert ts.Rope(inv_freq=f, pair_axis=[0, 1] * 16, num_axes=2).c.rotary_dim == 64
    for kw in (dict(inv_freq=f.double()), dict(inv_freq=torch.ones(64)[::2]), dict(inv_freq=f, pair_axis=[0]), dict(inv_freq=torch.ones(65)),
               dict(inv_freq=f, pair_axis=[300] * 32)):
        with pytest.raises(ValueError):
            ts.Rope(**kw)
    assert ts.rope_axes([2, 1, 1]) == [0, 0, 1, 2] and ts.rope_axes([3, 1, 2], dealt=True) == [0, 1, 2, 0, 2, 0] and ts.rope_axes([]) == []
    z = torch.zeros(4, dtype=torch.int32)
    p = ts.Problem(batch=1, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=9, dtype=ts.TS_F32, k_pool=z, v_pool=z,
                   page_indptr=z, page_indices=z, seq_lens=z)
    q, k = torch.zeros(3, 4, 64), torch.zeros(3, 2, 64)
    for bad in (dict(q=torch.zeros(3, 64, 4).transpose(1, 2)), dict(q=torch.zeros(3, 5, 64)), dict(k=torch.zeros(3, 256)[:, ::2]),
                dict(q_out=torch.zeros(3, 512)[:, :256])):
        a = dict(q=q, k=k, v=k, q_out=torch.zeros(3, 4, 64))
        a.update(bad)
        with pytest.raises(ValueError):
            ts.ts_rope_append(p, None, a["q"], a["k"], a["v"], z, 3, None, a["q_out"])


# ---------------------------------------------------------------------------------------------------------------------

def check(pool, seqs):
    """Every page is held by as many sequences as its count says, the free ones by none, and each sequence has just its pages."""
    held = np.zeros(pool.num_pages, int)
    for s in seqs:
        assert len(pool.pages(s)) == -(-pool.length(s) // pool.page_size)
        assert len(set(pool.pages(s))) == len(pool.pages(s))
        held[pool.pages(s)] += 1
    assert np.array_equal(held, pool.refs) and pool.free_pages == int((held == 0).sum()) and len(pool) == len(seqs)


def test_page_pool_against_contents():
    """Random adds, growths, forks, frees, replacements and gathers; a list of values per page stands for its contents."""
    for seed in range(30):
        rng = np.random.default_rng(seed)
        P, NP = int(rng.integers(1, 6)), int(rng.integers(6, 40))
        pool, store, want, names = PagePool(NP, P), np.zeros((NP, 6), int), {}, iter(range(10000))

        def copy(copies):
            assert not {a for a, _ in copies} & {b for _, b in copies}
            for a, b in copies:
                store[b] = store[a]

        def write(s, at):
            for t in range(at, pool.length(s)):
                store[pool.pages(s)[t // P], t % P] = want[s][t]

        for _ in range(120):
            what = rng.choice(["add", "grow", "grow", "grow", "fork", "free", "replace", "gather"])
            seqs = list(want)
            s = seqs[int(rng.integers(len(seqs)))] if seqs else None
            before = (pool.refs.copy(), pool.free_pages, {x: (pool.pages(x), pool.length(x)) for x in seqs})
            try:
                if what == "add":
                    name, n = next(names), int(rng.integers(0, 9))
                    pool.add(name, n)
                    want[name] = rng.integers(1, 1 << 30, n).tolist()
                    write(name, 0)
                elif what == "gather":
                    copy(pool.gather())
                    assert all(page < int((pool.refs > 0).sum()) for x in seqs for page in pool.pages(x))
                elif s is None:
                    continue
                elif what == "grow":
                    n = int(rng.integers(0, 7))
                    at = pool.length(s)
                    copy(pool.grow(s, n))
                    want[s] = want[s] + rng.integers(1, 1 << 30, n).tolist()
                    write(s, at)
                elif what == "fork":
                    name = next(names)
                    pool.fork(s, name)
                    want[name] = list(want[s])
                elif what == "free":
                    pool.free(s)
                    del want[s]
                else:
                    keep = sorted(rng.permutation(len(want[s]))[:int(rng.integers(0, len(want[s]) + 1))].tolist())
                    pages = pool.spare(len(keep) + int(rng.integers(0, 3)))
                    for j, t in enumerate(keep):
                        store[pages[j // P], j % P] = want[s][t]
                    if rng.random() < 0.2:
                        pool.give_back(pages)
                    else:
                        pool.replace(s, pages, len(keep))
                        want[s] = [want[s][t] for t in keep]
            except MemoryError:
                assert np.array_equal(before[0], pool.refs) and before[1] == pool.free_pages
                assert before[2] == {x: (pool.pages(x), pool.length(x)) for x in seqs}
            check(pool, list(want))
            for x, values in want.items():
                assert [store[pool.pages(x)[t // P], t % P] for t in range(pool.length(x))] == values, (seed, x)


def test_page_pool_table_and_refusals():
    pool = PagePool(10, 4)
    pool.add("a", 9)
    pool.add("b")
    ind, pages, lens = pool.table(["b", "a"], room=1)
    assert ind.tolist() == [0, 1, 5] and pages.tolist() == [0, 0, 1, 2, 0] and lens.tolist() == [0, 9] and ind.dtype == pages.dtype == lens.dtype == np.int32
    assert pool.table([])[1].size == 1
    for call, error in ((lambda: pool.add("a"), KeyError), (lambda: pool.fork("a", "b"), KeyError), (lambda: pool.free("x"), KeyError),
                        (lambda: pool.grow("x"), KeyError), (lambda: pool.grow("a", -1), ValueError), (lambda: pool.add("c", -1), ValueError),
                        (lambda: pool.add("c", 100), MemoryError), (lambda: pool.grow("a", 100), MemoryError),
                        (lambda: pool.spare(100), MemoryError), (lambda: pool.replace("a", [], 1), ValueError), (lambda: PagePool(0, 4), ValueError)):
        with pytest.raises(error):
            call()
    check(pool, ["a", "b"])


def test_spare_pages_stay_where_the_caller_knows_them():
    pool = PagePool(16, 4)
    pool.add("a", 12)                               # 0, 1, 2
    pool.add("b", 8)                                # 3, 4
    spare = pool.spare(7)                           # 5, 6
    pool.add("c", 12)                               # 7, 8, 9
    pool.free("a")
    moved = pool.gather()
    assert moved == [(9, 0), (8, 1), (7, 2)] and pool.pages("c") == [2, 1, 0] and pool.pages("b") == [3, 4]
    assert all(pool.refs[page] == 1 for page in spare)
    for wrong in ([0], [spare[0], spare[0]], [15]):
        with pytest.raises(ValueError):
            pool.give_back(wrong)
        with pytest.raises(ValueError):
            pool.replace("b", wrong, 1)
    assert pool.free_pages == 9 and pool.pages("b") == [3, 4]
    pool.replace("b", spare, 3)                     # 3, 4 and the second spare page come back
    assert pool.pages("b") == [spare[0]] and pool.free_pages == 12
    with pytest.raises(ValueError):
        pool.give_back(spare)                       # no longer spare
    assert pool.gather() == [(5, 3)] and pool.pages("b") == [3] and pool.pages("c") == [2, 1, 0]
