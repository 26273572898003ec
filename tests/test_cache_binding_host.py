"""What the binding of the cache's calls refuses before anything is launched: tensors whose layout or type the library cannot see."""
import pytest

import paper_2411_02886_amd as ts

torch = pytest.importorskip("torch")


def problem(dtype=None, **kw):
    z = torch.zeros(4, dtype=torch.int32)
    args = dict(batch=1, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=9, dtype=ts.TS_F32 if dtype is None else dtype,
                k_pool=z, v_pool=z, page_indptr=z, page_indices=z, seq_lens=z)
    args.update(kw)
    return ts.Problem(**args)


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_rows_that_overlap_are_refused(what):
    """Stride 0 would be taken as packed: rows would be read behind the one that is there."""
    ind = torch.zeros(2, dtype=torch.int32)
    heads = dict(q=4, k=2, v=2)
    for shape in ((3, heads[what], 64), (3, heads[what] * 64)):
        a = {n: torch.zeros(3, h, 64) for n, h in heads.items()}
        for bad in (torch.zeros(1, *shape[1:]).expand(*shape), torch.zeros(3 * 64 * 8).as_strided(shape, (64,) + ((64, 1) if len(shape) == 3 else (1,)))):
            a[what] = bad
            with pytest.raises(ValueError):
                ts.ts_rope_append(problem(), None, a["q"], a["k"], a["v"], ind, 3, None, torch.zeros(3, 4, 64))


def test_compact_refuses_new_lengths_in_the_place_of_what_it_reads():
    """The old lengths are read by many workgroups while one writes the new ones."""
    import ctypes

    from paper_2411_02886_amd.binding import _CProblem
    at = dict(k_pool=0x100000, v_pool=0x200000, page_indptr=0x300000, page_indices=0x400000, seq_lens=0x500000)
    p = _CProblem(batch=6, chunk=1, num_q_heads=8, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=4096, dtype=ts.TS_BF16, num_initial=0,
                  num_local=0, **at)
    idx, count, skip, to_indptr, to = 0x600000, 0x700000, 0x800000, 0x900000, 0xa00000
    for lens in (0x500000, 0x500000 + 20, 0x500000 - 20, count, count + 4, idx, idx + 6 * 4 * 4 - 4, 0x300000 + 24, to_indptr + 24, to_indptr - 4, skip + 4):
        assert ts.load().ts_cache_compact(ctypes.byref(p), idx, 4, count, skip, to_indptr, to, lens, None) == -1, hex(lens)


def test_copies_that_follow_each_other_are_cut_into_runs():
    import numpy as np

    from paper_2411_02886_amd.pages import PagePool, copy_runs
    assert copy_runs([]) == [] and copy_runs([(1, 2), (1, 3), (4, 5)]) == [(0, 3)] and copy_runs([(7, 7)]) == [(0, 1)]
    assert copy_runs([(5, 9), (9, 10)]) == [(0, 1), (1, 2)]                # reads what the first wrote
    assert copy_runs([(5, 9), (3, 5)]) == [(0, 1), (1, 2)]                 # overwrites what the first reads
    assert copy_runs([(5, 9), (9, 9), (4, 9)]) == [(0, 2), (2, 3)]         # writes the same page
    rng = np.random.default_rng(0)
    for _ in range(200):
        copies = [tuple(int(x) for x in rng.integers(0, 9, 2)) for _ in range(int(rng.integers(0, 14)))]
        want, got = np.arange(9), np.arange(9)
        for a, b in copies:
            want[b] = want[a]
        at = 0
        for begin, end in copy_runs(copies):
            assert begin == at and end > begin
            at = end
            src, dst = [a for a, _ in copies[begin:end]], [b for _, b in copies[begin:end]]
            pairs = {(a, b) for a, b in copies[begin:end] if a != b}
            assert len({b for _, b in pairs}) == len([1 for a, b in copies[begin:end] if a != b]) and not {a for a, _ in pairs} & {b for _, b in pairs}
            before = got.copy()
            for a, b in zip(src, dst):
                got[b] = before[a] if a != b else got[b]
        assert at == len(copies) and np.array_equal(want, got)
    # a fork grows, its own fork grows: the second copy reads what the first one wrote
    pool = PagePool(8, 4)
    pool.add("a", 2)
    pool.fork("a", "b")
    copies = pool.grow("b")
    pool.fork("b", "c")
    copies += pool.grow("c")
    assert copies == [(0, 1), (1, 2)] and copy_runs(copies) == [(0, 1), (1, 2)]


def test_a_list_of_copies_goes_where_the_pools_are(monkeypatch):
    from paper_2411_02886_amd import runtime
    calls = []
    monkeypatch.setattr(runtime.ts, "ts_pages_copy", lambda p, src, dst, n, pages: calls.append((src, dst, n, pages)))
    runtime.copy_pages(problem(), [(0, 1), (1, 2), (0, 3)], 9)
    assert [(a.tolist(), b.tolist(), n, pages) for a, b, n, pages in calls] == [([0], [1], 1, 9), ([1, 0], [2, 3], 2, 9)]
    assert all(t.device.type == "cpu" and t.is_contiguous() and t.dtype == torch.int32 for a, b, _, _ in calls for t in (a, b))
    runtime.copy_pages(None, [], 9)


def ints(*shape):
    return torch.zeros(*shape, dtype=torch.int32)


def attend(p, **kw):
    a = dict(q=torch.zeros(3, 4, 64), ind=ints(2), out=torch.zeros(3, 4, 64), lse=torch.zeros(3, 4), ws=torch.zeros(1 << 10))
    a.update(kw)
    for call in (ts.ts_paged_attn, ts.ts_paged_attn_rounded):
        call(p, a["q"], a["ind"], 3, 0, 0.1, a["out"], a["lse"], a["ws"])


def append(p, rope=None, **kw):
    a = dict(q=torch.zeros(3, 4, 64), k=torch.zeros(3, 2, 64), v=torch.zeros(3, 128), ind=ints(2), pos=None, q_out=torch.zeros(3, 4, 64))
    a.update(kw)
    ts.ts_rope_append(p, rope, a["q"], a["k"], a["v"], a["ind"], 3, a["pos"], a["q_out"])


def copy(p, n=2, pages=1, **kw):
    a = dict(src=ints(2), dst=ints(2))
    a.update(kw)
    ts.ts_pages_copy(p, a["src"], a["dst"], n, pages)


def compact(p, stride=4, **kw):
    a = dict(idx=ints(1, 4), count=ints(1), skip=None, to_indptr=ints(2), to_indices=ints(3), to_lens=ints(1))
    a.update(kw)
    ts.ts_cache_compact(p, a["idx"], stride, a["count"], a["skip"], a["to_indptr"], a["to_indices"], a["to_lens"])


WRONG_TYPES = [(attend, n) for n in ("q", "ind", "out", "lse")] + [(append, n) for n in ("q", "k", "v", "ind", "pos", "q_out")] + \
    [(copy, n) for n in ("src", "dst")] + [(compact, n) for n in ("idx", "count", "skip", "to_indptr", "to_indices", "to_lens")]
NAMES = dict(ind="q_indptr", pos="positions")


@pytest.mark.parametrize("call,name", WRONG_TYPES, ids=lambda x: getattr(x, "__name__", x))
def test_types_lengths_and_gaps_are_looked_at(call, name):
    """A torch int64 tensor is what cumsum and arange give; it would be read as pairs of int32."""
    z = torch.zeros(16 * 128)
    p = problem(k_pool=z, v_pool=z)
    rope = dict(rope=ts.Rope(inv_freq=torch.ones(32))) if call is append else {}
    whole = dict(q=(3, 4, 64), out=(3, 4, 64), q_out=(3, 4, 64), k=(3, 2, 64), v=(3, 2, 64), lse=(3, 4), ind=(2,), pos=(1, 3), src=(2,), dst=(2,), idx=(1, 4),
                 count=(1,), skip=(1,), to_indptr=(2,), to_indices=(1,), to_lens=(1,))[name]
    right = torch.float32 if len(whole) == 3 or name == "lse" else torch.uint8 if name == "skip" else torch.int32
    for wrong in {torch.int64, torch.float64, torch.float16, torch.bfloat16, torch.float32} - {right}:
        with pytest.raises(ValueError, match=NAMES.get(name, name)):
            call(p, **rope, **{name: torch.zeros(*whole, dtype=wrong)})
    with pytest.raises(ValueError, match=NAMES.get(name, name)):           # too short
        call(p, **rope, **{name: torch.zeros(*whole, dtype=right)[:-1] if whole != (1, 3) else torch.zeros(1, 2, dtype=right)})
    if len(whole) != 3 or name in ("out", "q_out"):
        if max(whole) > 1:
            with pytest.raises(ValueError, match=NAMES.get(name, name)):   # with gaps
                call(p, **rope, **{name: torch.zeros(*whole, 2, dtype=right)[..., 0]})
    with pytest.raises(ValueError, match="not on a GPU"):                  # all as it should be: pools in host memory are refused
        call(p, **rope)


def test_bf16_travels_as_such_or_as_bits():
    z = torch.zeros(16 * 128, dtype=torch.bfloat16)
    p = problem(ts.TS_BF16, k_pool=z, v_pool=z)
    for dtype in (torch.bfloat16, torch.int16):
        x = torch.zeros(3, 4, 64, dtype=dtype)
        with pytest.raises(ValueError, match="not on a GPU"):
            attend(p, q=x, out=x.clone())
    for dtype in (torch.float16, torch.float32):
        with pytest.raises(ValueError, match="^q"):
            attend(p, q=torch.zeros(3, 4, 64, dtype=dtype))


def test_more_pages_than_the_pools_hold_are_refused():
    z = torch.zeros(2, 16, 2, 64)
    with pytest.raises(ValueError, match="num_pages"):
        copy(problem(k_pool=z, v_pool=z), pages=3)
    with pytest.raises(ValueError, match="num_pages"):
        copy(problem(k_pool=z, v_pool=z[:1]), pages=2)
    with pytest.raises(ValueError, match="not on a GPU"):
        copy(problem(k_pool=z, v_pool=None), pages=2)


class FakeLayer:
    """What attend_all and append need of a layer, with calls that are written down instead of launched."""

    def __init__(self, monkeypatch, B=2, C=1):
        from paper_2411_02886_amd import runtime
        self.calls, self.stream, self.bytes = [], 7, 1 << 12
        fake, ts0 = self, runtime.ts

        class Layer(runtime._NewTokens):
            def __init__(self):
                z = ints(9)
                self.k_pool, self.B, self.D = torch.zeros(4, 16, 2, 64), B, 64
                self.problem = ts.Problem(batch=B, chunk=C, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=64, dtype=ts.TS_F32,
                                          k_pool=self.k_pool, v_pool=self.k_pool, page_indptr=z, page_indices=z, seq_lens=z)
                self.out, self.lse = torch.zeros(B, C, 4, 64), torch.zeros(B, C, 4)

        for name in ("ts_paged_attn", "ts_paged_attn_rounded", "ts_rope_append"):
            monkeypatch.setattr(ts0, name, lambda *a, name=name: fake.calls.append((name,) + a))
        monkeypatch.setattr(ts0, "ts_paged_attn_workspace_bytes", lambda p, rows: fake.bytes * p.c.chunk)
        monkeypatch.setattr(ts0, "_current_stream", lambda: fake.stream)
        self.layer = Layer()


def test_each_stream_has_a_workspace_of_its_own_and_none_is_replaced(monkeypatch):
    f = FakeLayer(monkeypatch)
    q = torch.zeros(2, 1, 4, 64)
    ws = []
    for stream, size in ((7, 1 << 12), (8, 1 << 12), (7, 1 << 14), (7, 1 << 12), (8, 1 << 12)):
        f.stream, f.bytes = stream, size
        f.layer.attend_all(q)
        ws.append(f.calls[-1][9])
        assert ws[-1].numel() * 4 >= size
    at = [w.data_ptr() for w in ws]
    assert len({at[0], at[1], at[2]}) == 3 and at[3] == at[0] and at[4] == at[1]
    own = torch.zeros(1 << 12)
    f.layer.attend_all(q, ws=own)
    assert f.calls[-1][9] is own
    g = FakeLayer(monkeypatch)                      # another layer, another workspace
    g.layer.attend_all(q)
    assert g.calls[-1][9].data_ptr() not in at


def test_append_takes_the_shapes_that_attend_all_takes(monkeypatch):
    f = FakeLayer(monkeypatch, B=2, C=3)
    q, k = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64)
    f.layer.append(k, k, q=q, q_out=torch.zeros_like(q))
    _, _, _, q1, k1, v1, _, rows, _, _ = f.calls[-1]
    assert rows == 6 and tuple(q1.shape) == (6, 4, 64) and tuple(k1.shape) == tuple(v1.shape) == (6, 2, 64) and q1.data_ptr() == q.data_ptr()
    f.layer.append(None, None, q=q, q_out=q)
    assert f.calls[-1][7] == 6
    fused = torch.zeros(2, 3, 8, 64)                # parts of a projection stay views
    f.layer.append(fused[:, :, 4:6], fused[:, :, 6:], q=fused[:, :, :4], q_out=q)
    assert [t.data_ptr() - fused.data_ptr() for t in f.calls[-1][3:6]] == [0, 4 * 256, 6 * 256] and f.calls[-1][4].stride(0) == 512
    f.layer.append(k.view(6, 128), k.view(6, 128))  # rows as before
    assert f.calls[-1][7] == 6 and f.calls[-1][4].dim() == 2


def test_packed_rows_may_say_how_many_a_sequence_has(monkeypatch):
    f = FakeLayer(monkeypatch)
    lay, q, ind = f.layer, torch.zeros(40, 4, 64), ints(3)
    for most in (40, 16, 40):
        lay.attend_all(q, q_indptr=ind, out=q.clone(), most_new=most)
        p, ws = f.calls[-1][1], f.calls[-1][9]
        assert p.c.chunk == most and ws.numel() * 4 >= f.bytes * most and f.calls[-1][4] == 40
        assert [getattr(p.c, n) for n, _ in p.c._fields_ if n != "chunk"] == [getattr(lay.problem.c, n) for n, _ in p.c._fields_ if n != "chunk"]
    assert f.calls[0][1] is f.calls[2][1] and lay.problem.c.chunk == 1
    lay.attend_all(q, q_indptr=ind, out=q.clone())
    assert f.calls[-1][1] is lay.problem
    lay.problem = lay.problem.with_chunk(1)         # another pool: the kept ones are dropped
    lay.attend_all(q, q_indptr=ind, out=q.clone(), most_new=40)
    assert f.calls[-1][1] is not f.calls[0][1]
    lay.attend_all(torch.zeros(2, 1, 4, 64), most_new=40)       # a step's own rows: the layer's chunk
    assert f.calls[-1][1] is lay.problem


def test_a_negative_number_of_spare_tokens_is_refused():
    from paper_2411_02886_amd.pages import PagePool
    pool = PagePool(4, 4)
    with pytest.raises(ValueError):
        pool.spare(-5)
    assert pool.spare(0) == [] and pool.free_pages == 4


def test_the_rounded_form_refuses_what_the_other_does(monkeypatch):
    import test_cache_host
    lib = ts.load()

    class Rounded:
        ts_paged_attn = staticmethod(lib.ts_paged_attn_rounded)

    with monkeypatch.context() as m:
        m.setattr(test_cache_host.ts, "load", lambda: Rounded)
        test_cache_host.test_paged_attn_refusals()
