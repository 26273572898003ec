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


CALLS = [(b_append, n) for n in ("q", "k", "v", "ind", "pos", "q_out")] + [(b_read, n) for n in ("ind", "k_out", "v_out")] + [(b_copy, n) for n in ("src", "dst")]


@pytest.mark.parametrize("call,name", CALLS, ids=lambda x: getattr(x, "__name__", x))
def test_wrong_types_lengths_and_devices_are_refused(call, name):
    c = ts.QuantCache(**parts())
    bad = torch.zeros(3, 4, 64, dtype=torch.float64)
    with pytest.raises(ValueError):
        call(problem(), c, **{name: bad})
    if name not in ("pos",):
        with pytest.raises(ValueError):
            call(problem(), c, **{name: ints(1)[:0] if name in ("ind", "src", "dst") else torch.zeros(1, 2, 64)})
    with pytest.raises(ValueError, match="not on a GPU"):
        call(problem(), c)
    for p in (problem(page_size=8), problem(head_dim=128), problem(num_kv_heads=4)):
        with pytest.raises(ValueError, match="the cache has pages"):
            call(p, c)


def test_more_pages_than_the_cache_holds_are_refused():
    with pytest.raises(ValueError, match="holds 3"):
        ts.ts_quant_pages_copy(problem(), ts.QuantCache(**parts()), ints(1), ints(1), 1, 4)
