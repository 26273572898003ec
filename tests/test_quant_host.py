"""What the calls on the 8-bit cache and on drafted trees refuse, in the library and in the binding, before anything is launched."""
import ctypes

import pytest

import paper_2411_02886_amd as ts
from paper_2411_02886_amd.binding import _CProblem, _CQuant, _CRope

torch = pytest.importorskip("torch")
A, BIG = 0x10000, 1 << 40
OK, BAD, UNSUP, WS = 0, -1, -2, -3


def cproblem(**kw):
    base = dict(batch=2, chunk=1, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=4096, dtype=ts.TS_BF16,
                k_pool=None, v_pool=None, page_indptr=A, page_indices=A, seq_lens=A, num_initial=0, num_local=0)
    base.update(kw)
    return ctypes.byref(_CProblem(**base))


def cquant(**kw):
    base = dict(k_codes=0x8000000, v_codes=0x9000000, k_scale=0xa000000, v_scale=0xb000000, code=ts.TS_INT8)
    base.update(kw)
    return ctypes.byref(_CQuant(**base))


BAD_QUANT = [None] + [cquant(**kw) for kw in (dict(k_codes=None), dict(v_codes=None), dict(k_scale=None), dict(v_scale=None), dict(code=2), dict(code=-1),
                                              dict(k_codes=0x8000008), dict(v_codes=1), dict(k_scale=0xa000004), dict(v_scale=0xb000008))]


def rope(**kw):
    base = dict(inv_freq=A, rotary_dim=64, num_axes=1, adjacent=0, scale=1.0)
    axes = kw.pop("pair_axis", [0] * 64)
    base.update(kw)
    return ctypes.byref(_CRope(**base, pair_axis=(ctypes.c_uint8 * 64)(*axes)))


def append(p=None, c=None, r=None, q=A, qs=0, k=0x200000, ks=0, v=0x300000, vs=0, ind=None, rows=2, pos=None, out=0x900000, quant=True):
    return ts.load().ts_quant_append(p or cproblem(), (c or cquant()) if quant else None, r, q, qs, k, ks, v, vs, ind, rows, pos, out, None)


def test_append_refusals():
    for r in (dict(rotary_dim=63), dict(rotary_dim=66), dict(rotary_dim=-2), dict(num_axes=0), dict(num_axes=5), dict(adjacent=2),
              dict(scale=float("nan")), dict(scale=float("inf")), dict(inv_freq=None), dict(pair_axis=[0] * 31 + [1] + [0] * 32)):
        assert append(r=rope(**r)) == BAD, r
    for kw in (dict(q=None), dict(out=None), dict(k=None), dict(v=None), dict(k=None, v=None), dict(rows=3), dict(rows=-2),
               dict(q=A + 4), dict(out=0x900002), dict(k=0x200008), dict(v=0x300001), dict(qs=500), dict(qs=516), dict(ks=100), dict(ks=132),
               dict(vs=-128), dict(out=A + 1024), dict(q=A, out=A, qs=1024), dict(out=0x200000), dict(out=0x300000 - 64),
               dict(p=cproblem(seq_lens=None)), dict(p=cproblem(num_q_heads=7)), dict(quant=False)):
        assert append(r=rope(), **kw) == BAD, kw
    for c in BAD_QUANT[1:]:
        assert append(c=c) == BAD
    assert append(p=cproblem(head_dim=32)) == UNSUP
    assert append(rows=0, q=None, out=None, k=None, v=None) == OK


def read(p=None, c=None, ind=None, rows=2, k=0x200000, v=0x300000, quant=True):
    return ts.load().ts_quant_read(p or cproblem(), (c or cquant()) if quant else None, ind, rows, k, v, None)


def test_read_refusals():
    for kw in (dict(k=None, v=None), dict(k=0x200008), dict(v=0x300004), dict(rows=3), dict(rows=-1), dict(quant=False), dict(v=0x200000 + 256),
               dict(p=cproblem(page_indptr=None))):
        assert read(**kw) == BAD, kw
    for c in BAD_QUANT[1:]:
        assert read(c=c) == BAD
    assert read(p=cproblem(page_size=12)) == UNSUP
    assert read(rows=0, k=None, v=None) == OK


def test_pages_copy_refusals():
    call = lambda p=None, c=None, src=A, dst=0x20000, n=3, pages=9: ts.load().ts_quant_pages_copy(p or cproblem(), c or cquant(), src, dst, n, pages, None)
    for kw in (dict(src=None), dict(dst=None), dict(n=-1), dict(pages=0)):
        assert call(**kw) == BAD, kw
    for c in BAD_QUANT[1:]:
        assert call(c=c) == BAD
    assert call(p=cproblem(head_dim=96)) == UNSUP
    assert call(n=0, src=None, dst=None) == OK


def attn(p=None, c=None, q=A, ind=None, rows=2, window=0, mask=None, words=0, sm=0.1, out=0x900000, lse=None, ws=0x2000000, ws_bytes=BIG, quant=True):
    return ts.load().ts_quant_attn(p or cproblem(), (c or cquant()) if quant else None, q, ind, rows, window, mask, words, sm, out, lse, ws, ws_bytes, None)


def test_attn_refusals():
    for kw in (dict(q=None), dict(out=None), dict(rows=3), dict(rows=-1), dict(window=-1), dict(sm=float("nan")), dict(sm=float("inf")), dict(quant=False),
               dict(mask=0x500000), dict(mask=0x500000, words=-1), dict(mask=0x500002, words=1), dict(q=A + 8), dict(out=0x900004), dict(out=A),
               dict(out=A + 2 * 8 * 64 * 2 - 16), dict(p=cproblem(seq_lens=None)), dict(p=cproblem(num_q_heads=7))):
        assert attn(**kw) == BAD, kw
    for c in BAD_QUANT[1:]:
        assert attn(c=c) == BAD
    assert attn(p=cproblem(head_dim=96)) == UNSUP and attn(p=cproblem(page_size=12)) == UNSUP
    for kw in (dict(ws=None), dict(ws=0x2000010), dict(ws_bytes=16)):
        assert attn(**kw) == WS, kw
    assert attn(rows=0, q=None, out=None, ws=None, ws_bytes=0) == OK


def test_attn_workspace():
    L, out = ts.load(), ctypes.c_size_t(0)
    get = lambda rows, **kw: (L.ts_quant_attn_workspace_bytes(cproblem(**kw), rows, ctypes.byref(out)), out.value)
    assert get(-1)[0] == BAD and L.ts_quant_attn_workspace_bytes(None, 1, ctypes.byref(out)) == BAD
    assert get(1, head_dim=80)[0] == UNSUP
    for dtype in (ts.TS_BF16, ts.TS_F32):                     # one workspace serves every call with fewer rows, shorter chunks and sequences, fewer sequences
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


def tree_mask(p=None, parents=A, ind=None, rows=2, mask=0x200000, words=3, pos=0x300000):
    return ts.load().ts_tree_mask(p or cproblem(), parents, ind, rows, mask, words, pos, None)


def test_tree_mask_refusals():
    for kw in (dict(parents=None), dict(mask=None), dict(words=0), dict(words=-1), dict(rows=3), dict(rows=-1), dict(mask=A + 4), dict(pos=A), dict(pos=0x200000 + 20),
               dict(mask=A - 8), dict(p=cproblem(seq_lens=None)), dict(p=cproblem(seq_lens=0x200004))):
        assert tree_mask(**kw) == BAD, kw
    assert tree_mask(p=cproblem(head_dim=80)) == UNSUP
    assert tree_mask(rows=0, parents=None, mask=None, pos=None) == OK


def tree_attn(p=None, q=A, ind=None, rows=2, window=0, mask=0x500000, words=1, sm=0.1, out=0x900000, lse=None, ws=0x2000000, ws_bytes=BIG):
    return ts.load().ts_tree_attn(p or cproblem(k_pool=A, v_pool=A), q, ind, rows, window, mask, words, sm, out, lse, ws, ws_bytes, None)


def test_tree_attn_refusals():
    pools = dict(k_pool=A, v_pool=A)
    for kw in (dict(q=None), dict(out=None), dict(rows=3), dict(rows=-1), dict(window=-1), dict(sm=float("nan")), dict(sm=float("inf")),
               dict(mask=None), dict(mask=0x500002), dict(words=0), dict(words=-4),
               dict(q=A + 8), dict(out=0x900004), dict(out=A), dict(p=cproblem()), dict(p=cproblem(**dict(pools, v_pool=None))),
               dict(p=cproblem(**dict(pools, k_pool=A + 2))), dict(p=cproblem(**pools, seq_lens=None))):
        assert tree_attn(**kw) == BAD, kw
    assert tree_attn(p=cproblem(**pools, head_dim=96)) == UNSUP
    for kw in (dict(ws=None), dict(ws=0x2000010), dict(ws_bytes=16)):
        assert tree_attn(**kw) == WS, kw
    assert tree_attn(rows=0, q=None, out=None, mask=None, ws=None, ws_bytes=0) == OK


def keep(p=None, c=None, path=0x500000, stride=4, count=0x600000, ind=None, to=0x700000):
    return ts.load().ts_tree_keep(p or cproblem(k_pool=0x100000, v_pool=0x200000), c, path, stride, count, ind, to, None)


def test_tree_keep_refusals():
    for kw in (dict(path=None), dict(count=None), dict(to=None), dict(stride=0), dict(p=cproblem()), dict(p=cproblem(k_pool=A)), dict(p=cproblem(k_pool=A + 4, v_pool=A)),
               dict(to=A), dict(to=A + 4), dict(to=A - 4), dict(to=0x500000 + 2 * 4 * 4 - 4), dict(to=0x600004), dict(ind=0x700004), dict(ind=0x700000 - 8)):
        assert keep(**kw) == BAD, kw
    for c in BAD_QUANT[1:]:
        assert keep(c=c) == BAD
    assert keep(p=cproblem(k_pool=A, v_pool=A, page_size=12)) == UNSUP


# ---- the binding

def problem(**kw):
    z = torch.zeros(4, dtype=torch.int32)
    args = dict(batch=1, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=9, dtype=ts.TS_F32, k_pool=None, v_pool=None, page_indptr=z,
                page_indices=z, seq_lens=z)
    args.update(kw)
    return ts.Problem(**args)


def parts(**kw):
    a = dict(k_codes=torch.zeros(3, 16, 2, 64, dtype=torch.uint8), v_codes=torch.zeros(3, 16, 2, 64, dtype=torch.uint8), k_scale=torch.zeros(3, 2, 16),
             v_scale=torch.zeros(3, 2, 16), format=ts.TS_INT8)
    a.update(kw)
    return a


def test_a_cache_is_made_of_tensors_that_fit():
    ts.QuantCache(**parts())
    ts.QuantCache(**parts(k_codes=torch.zeros(3, 16, 2, 64, dtype=torch.int8)))
    ts.QuantCache(**parts(format=ts.TS_E4M3, k_codes=torch.zeros(3, 16, 2, 64).to(torch.float8_e4m3fn)))
    assert ts.QuantCache.empty(3, 16, 2, 64, ts.TS_E4M3, device="cpu").shape == (16, 2, 64)
    for kw in (dict(format=2), dict(k_codes=torch.zeros(3, 16, 2, 64)), dict(format=ts.TS_E4M3, v_codes=torch.zeros(3, 16, 2, 64, dtype=torch.int8)),
               dict(k_codes=torch.zeros(3, 16, 2, 64).to(torch.float8_e4m3fn)), dict(k_scale=torch.zeros(3, 16, 2)), dict(v_scale=torch.zeros(2, 2, 16)),
               dict(v_codes=torch.zeros(4, 16, 2, 64, dtype=torch.uint8)), dict(k_scale=torch.zeros(3, 2, 16, dtype=torch.float64)),
               dict(k_codes=torch.zeros(3, 2, 16, 64, dtype=torch.uint8).transpose(1, 2)), dict(k_scale=torch.zeros(3 * 2 * 16))):
        with pytest.raises(ValueError):
            ts.QuantCache(**parts(**kw))


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def b_append(p, c, **kw):
    a = dict(q=torch.zeros(3, 4, 64), k=torch.zeros(3, 2, 64), v=torch.zeros(3, 128), ind=ints(2), pos=None, q_out=torch.zeros(3, 4, 64))
    a.update(kw)
    ts.ts_quant_append(p, c, None, a["q"], a["k"], a["v"], a["ind"], 3, a["pos"], a["q_out"])


def b_read(p, c, **kw):
    a = dict(ind=ints(2), k_out=torch.zeros(3, 2, 64), v_out=torch.zeros(3, 2, 64))
    a.update(kw)
    ts.ts_quant_read(p, c, a["ind"], 3, a["k_out"], a["v_out"])


def b_copy(p, c, **kw):
    a = dict(src=ints(2), dst=ints(2))
    a.update(kw)
    ts.ts_quant_pages_copy(p, c, a["src"], a["dst"], 2, 3)


def b_attn(p, c, **kw):
    a = dict(q=torch.zeros(3, 4, 64), ind=ints(2), mask=ints(3, 1), out=torch.zeros(3, 4, 64), lse=torch.zeros(3, 4))
    a.update(kw)
    ts.ts_quant_attn(p, c, a["q"], a["ind"], 3, 0, a["mask"], 0.1, a["out"], a["lse"], torch.zeros(64))


def b_mask(p, c, **kw):
    a = dict(parents=ints(3), ind=ints(2), mask=ints(3, 1), positions=ints(3))
    a.update(kw)
    ts.ts_tree_mask(p, a["parents"], a["ind"], 3, a["mask"], a["positions"])


def b_tree(p, c, **kw):
    a = dict(q=torch.zeros(3, 4, 64), ind=ints(2), mask=ints(3, 1), out=torch.zeros(3, 4, 64), lse=torch.zeros(3, 4))
    a.update(kw)
    ts.ts_tree_attn(p, a["q"], a["ind"], 3, 0, a["mask"], 0.1, a["out"], a["lse"], torch.zeros(64))


def b_keep(p, c, **kw):
    a = dict(path=ints(1, 4), count=ints(1), ind=ints(2), to_lens=ints(1))
    a.update(kw)
    ts.ts_tree_keep(p, c, a["path"], 4, a["count"], a["ind"], a["to_lens"])


SHAPED = ("b_append", "b_read", "b_copy", "b_keep", "b_attn")          # calls that compare the cache with the problem
CALLS = [(b_mask, n) for n in ("parents", "ind", "mask", "positions")] + [(b_tree, n) for n in ("q", "ind", "mask", "out", "lse")] + \
    [(b_attn, n) for n in ("q", "ind", "mask", "out", "lse")] + [(b_keep, n) for n in ("path", "count", "ind", "to_lens")] + [(b_append, n) for n in ("q", "k", "v", "ind", "pos", "q_out")] + [(b_read, n) for n in ("ind", "k_out", "v_out")] + [(b_copy, n) for n in ("src", "dst")]


@pytest.mark.parametrize("call,name", CALLS, ids=lambda x: getattr(x, "__name__", x))
def test_wrong_types_lengths_and_devices_are_refused(call, name):
    c = ts.QuantCache(**parts())
    bad = torch.zeros(3, 4, 64, dtype=torch.float64)
    with pytest.raises(ValueError):
        call(problem(), c, **{name: bad})
    if name not in ("pos",):
        short = ints(1)[:0] if name in ("ind", "src", "dst", "parents", "positions", "path", "count", "to_lens") else ints(1, 1) if name == "mask" else torch.zeros(1, 2, 64)
        with pytest.raises(ValueError):
            call(problem(), c, **{name: short[:, :1, :1] if name == "lse" else short})
    with pytest.raises(ValueError, match="not on a GPU"):
        call(problem(), c)
    for p in () if call.__name__ not in SHAPED else (problem(page_size=8), problem(head_dim=128), problem(num_kv_heads=4)):
        with pytest.raises(ValueError, match="the cache has pages"):
            call(p, c)


def test_more_pages_than_the_cache_holds_are_refused():
    with pytest.raises(ValueError, match="holds 3"):
        ts.ts_quant_pages_copy(problem(), ts.QuantCache(**parts()), ints(1), ints(1), 1, 4)


def test_a_sequence_is_cut():
    from paper_2411_02886_amd.pages import PagePool
    pool = PagePool(10, 4)
    pool.add("a", 18)                                    # five pages
    pool.fork("a", "b")
    with pytest.raises(ValueError):
        pool.cut("a", 19)
    with pytest.raises(ValueError):
        pool.cut("a", -1)
    pool.cut("a", 18)
    assert pool.pages("a") == [0, 1, 2, 3, 4] and pool.free_pages == 5
    pool.cut("a", 9)
    assert pool.pages("a") == [0, 1, 2] and pool.length("a") == 9 and pool.free_pages == 5 and pool.pages("b") == [0, 1, 2, 3, 4]
    assert pool.grow("a", 1) == [(2, 5)]                 # the page behind the cut is still b's
    pool.cut("b", 0)
    assert pool.pages("b") == [] and pool.free_pages == 10 - 3 and pool.length("b") == 0
    assert pool.grow("b", 2) == [] and pool.pages("b") == [2]


class Layer:
    """A layer whose calls are written down instead of launched."""

    def __init__(self, monkeypatch):
        from paper_2411_02886_amd import runtime
        self.calls, fake, z = [], self, torch.zeros(9, dtype=torch.int32)
        for name in ("ts_rope_append", "ts_quant_append", "ts_quant_read", "ts_tree_mask", "ts_tree_keep", "ts_paged_attn", "ts_paged_attn_rounded", "ts_tree_attn", "ts_quant_attn",
                     "ts_pages_copy", "ts_quant_pages_copy"):
            monkeypatch.setattr(runtime.ts, name, lambda *a, name=name: fake.calls.append((name,) + a))
        for name in ("ts_paged_attn_workspace_bytes", "ts_quant_attn_workspace_bytes"):
            monkeypatch.setattr(runtime.ts, name, lambda p, rows, name=name: 256 if name == "ts_paged_attn_workspace_bytes" else 512)
        monkeypatch.setattr(runtime.ts, "_current_stream", lambda: 7)

        class New(runtime._NewTokens):
            k_pool, B, D = torch.zeros(4, 16, 2, 64), 2, 64
            problem = ts.Problem(batch=2, chunk=3, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=64, dtype=ts.TS_F32, k_pool=k_pool, v_pool=k_pool,
                                 page_indptr=z, page_indices=z, seq_lens=z)
            out, lse = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 4)

        self.layer, self.copy_pages = New(), runtime.copy_pages


def test_a_layer_calls_what_its_arguments_say(monkeypatch):
    f = Layer(monkeypatch)
    lay, cache, ind = f.layer, ts.QuantCache.empty(4, 16, 2, 64, ts.TS_INT8, device="cpu"), torch.zeros(3, dtype=torch.int32)
    q, kv, mask = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros((6, 1), dtype=torch.int32)
    for kw, name in (({}, "ts_paged_attn"), (dict(round_weights=True), "ts_paged_attn_rounded"), (dict(mask=mask), "ts_tree_attn"), (dict(cache=cache), "ts_quant_attn"),
                     (dict(cache=cache, mask=mask), "ts_quant_attn")):
        lay.attend_all(q, window=5, **kw)
        call = f.calls[-1]
        at = 2 if "cache" in kw else 1
        assert call[0] == name and call[at + 1:at + 5] == (q, None, 6, 5) and ("cache" not in kw or call[2] is cache)
        assert call[-1].numel() * 4 == (512 if "cache" in kw else 256) and call[-3] is lay.out and call[-2] is lay.lse
        assert name not in ("ts_tree_attn", "ts_quant_attn") or call[at + 5] is kw.get("mask")
    for kw in (dict(mask=mask), dict(cache=cache)):
        with pytest.raises(ValueError, match="round_weights"):
            lay.attend_all(q, round_weights=True, **kw)
    lay.append(kv, kv, q=q, q_out=q, cache=cache)
    assert f.calls[-1][0] == "ts_quant_append" and f.calls[-1][2] is cache and f.calls[-1][8] == 6 and f.calls[-1][10] is q
    lay.append(kv, kv)
    assert f.calls[-1][0] == "ts_rope_append" and f.calls[-1][7] == 6
    rows = torch.zeros(11, 2, 64)
    lay.read_back(cache, rows, None, q_indptr=ind)
    assert f.calls[-1][:1] + f.calls[-1][2:] == ("ts_quant_read", cache, ind, 11, rows, None)
    lay.read_back(cache, None, rows)
    assert f.calls[-1][4] == 6
    parents = torch.zeros(11, dtype=torch.int32)
    lay.tree_mask(parents, mask, q_indptr=ind)
    assert f.calls[-1][:1] + f.calls[-1][2:] == ("ts_tree_mask", parents, ind, 11, mask, None)
    path = torch.zeros((2, 5), dtype=torch.int32)
    lay.keep(path, ind, ind, q_indptr=ind, cache=cache)
    assert f.calls[-1][:1] + f.calls[-1][2:] == ("ts_tree_keep", cache, path, 5, ind, ind, ind)
    f.copy_pages(lay.problem, [(0, 1), (1, 2)], 4, cache=cache)
    assert [c[0] for c in f.calls[-2:]] == ["ts_quant_pages_copy"] * 2 and f.calls[-1][2] is cache
    f.copy_pages(lay.problem, [(0, 1)], 4)
    assert f.calls[-1][0] == "ts_pages_copy"
