"""ts_paged_attn against the definition in 64 bits: lengths from nothing to thousands, packed and padded rows, windows, page sizes,
head layouts, rows that see nothing, neighbours full of NaN."""
import math

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


def workspace(ts, p, rows):
    n = ts.ts_paged_attn_workspace_bytes(p, rows)
    return torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")     # NaN in every word: nothing may be read first


def run(ts, cache, H, new, window=0, packed=True, sm=None, seed=0, max_seq_len=None, q_scale=1.0, behind=0, chunk=None):
    """(out, lse, reference); `behind` rows after the last sequence have to stay as they were."""
    from paper_2411_02886_amd.runtime import to_device, to_host
    D = cache.D
    sm = 1.0 / math.sqrt(D) if sm is None else sm
    T = sum(new) + behind
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    q = W.store(q_scale * rng.standard_normal((T, H, D), dtype=np.float32), cache.dtype)
    chunk = max(1, max(new)) if chunk is None else chunk
    p, _, _ = cache.problem(H, chunk=chunk, max_seq_len=max_seq_len)
    ind = to_device(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None
    es = torch.int16 if cache.dtype == BF else torch.float32
    out = torch.full((T, H, D), 77, dtype=es, device="cuda:0")
    lse = torch.full((T, H), 55.0, dtype=torch.float32, device="cuda:0")
    ts.ts_paged_attn(p, to_device(q), ind, T, window, sm, out, lse, workspace(ts, p, T))
    torch.cuda.synchronize()
    o, l = to_host(out, bits16=cache.dtype == BF), to_host(lse)
    if behind:
        assert np.all(o[T - behind:] == 77) and np.all(l[T - behind:] == 55.0)
    o = W.as_f32(o, cache.dtype).astype(np.float64)
    G = H // cache.H_kv
    ref = attention(cache, q[:T - behind], new, window, float(np.float32(sm)), [cache.dtype == BF and n * G > 32 for n in new])
    return o[:T - behind], l[:T - behind].astype(np.float64), ref


HEADS = [(1, 1), (8, 8), (8, 4), (6, 2), (8, 2), (10, 2), (6, 1), (28, 4), (16, 2), (32, 32)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_single_tokens_of_every_head_layout(gpu, dtype, D, H, H_kv):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 300, 1]
    c = Cache(dtype, H_kv, D, 16, lens, seed=H * 131 + D)
    o, l, ref = run(gpu, c, H, [1] * len(lens), packed=False, seed=H)
    check_attention(o, l, ref, "tokens")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_prompts_of_every_head_layout(gpu, dtype, D, H, H_kv):
    new, old = [65, 1, 70], [0, 40, 131]
    c = Cache(dtype, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H * 17 + D)
    o, l, ref = run(gpu, c, H, new, seed=H)
    check_attention(o, l, ref, "prompts")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 257])
def test_lengths_of_a_chunk(gpu, dtype, D, n):
    c = Cache(dtype, 2, D, 16, [n, n + 1, n + 63, n + 64, n + 200], seed=n)
    o, l, ref = run(gpu, c, 8, [n] * 5, packed=False, seed=n)
    check_attention(o, l, ref, n)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 2, 15, 63, 64, 65, 100, 128, 1 << 30])
@pytest.mark.parametrize("D", [64, 128])
def test_windows(gpu, dtype, window, D):
    new = [1, 90, 0, 5, 200]
    c = Cache(dtype, 2, D, 8, [300, 290, 17, 5, 517], seed=window % 1000)
    o, l, ref = run(gpu, c, 6, new, window=window, seed=3)
    check_attention(o, l, ref, window)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
def test_sequences_without_tokens_and_rows_that_see_nothing(gpu, dtype, D):
    # no tokens at all; more new tokens than the sequence holds (the first rows' places are negative); rows behind the last one
    new, lens = [0, 3, 70, 2, 0, 1, 40], [0, 0, 30, 2, 9, 0, 41]
    c = Cache(dtype, 4, D, 16, lens, seed=5)
    o, l, ref = run(gpu, c, 8, new, seed=5, behind=3)
    check_attention(o, l, ref, "empty")
    assert np.isneginf(l[:3]).all() and np.isneginf(l[3:43]).all() and np.isfinite(l[43:73]).all()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_nothing_to_do(gpu, dtype):
    c = Cache(dtype, 2, 64, 16, [5, 0], seed=1)
    p, _, _ = c.problem(8)
    from paper_2411_02886_amd.runtime import to_device
    gpu.ts_paged_attn(p, None, to_device(np.zeros(3, np.int32)), 0, 0, 0.1, None, None, None)
    torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("P", [1, 4, 8, 32, 64, 256])
@pytest.mark.parametrize("chunk", [1, 50])
def test_page_sizes(gpu, dtype, P, chunk):
    c = Cache(dtype, 2, 128, P, [chunk + 333, chunk + 64], seed=P)
    o, l, ref = run(gpu, c, 8, [chunk] * 2, packed=False, seed=P)
    check_attention(o, l, ref, P)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sm,q_scale", [(0.0, 1.0), (-0.3, 1.0), (1.0, 4.0), (64.0, 30.0)])
@pytest.mark.parametrize("n", [1, 60])
def test_scales_and_large_logits(gpu, dtype, sm, q_scale, n):
    # 64 * 30: logits of tens of thousands; a row is then its largest logit's value, and the bound, which grows with the logits, stays small
    c = Cache(dtype, 2, 64, 16, [n + 150, n + 40], seed=n, scale=q_scale)
    o, l, ref = run(gpu, c, 8, [n] * 2, packed=False, sm=sm, q_scale=q_scale, seed=n)
    check_attention(o, l, ref, (sm, q_scale))


@pytest.mark.parametrize("dtype,H,H_kv,D,lens", [(BF, 32, 8, 128, [9000, 3, 20001, 128, 5000]), (F32, 8, 2, 64, [6000, 1, 11000]),
                                                 (BF, 4, 4, 64, [12345]), (F32, 16, 4, 128, [5001, 70])])
@pytest.mark.parametrize("loose", [False, True], ids=["", "loose bound"])
def test_long_caches_are_cut_into_shares(gpu, dtype, H, H_kv, D, lens, loose):
    c = Cache(dtype, H_kv, D, 16, lens, seed=len(lens))
    o, l, ref = run(gpu, c, H, [1] * len(lens), packed=False, seed=9, max_seq_len=1 << 20 if loose else None)
    check_attention(o, l, ref, lens)


@pytest.mark.parametrize("dtype,H,H_kv,D", [(BF, 28, 4, 128), (BF, 8, 2, 64), (F32, 8, 2, 128)])
def test_single_tokens_beside_pieces_of_prompts(gpu, dtype, H, H_kv, D):
    new = [1, 300, 1, 0, 7, 64, 1, 9, 33]
    old = [4000, 0, 3, 50, 900, 1500, 0, 2000, 777]
    c = Cache(dtype, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=12)
    for window in (0, 500):
        o, l, ref = run(gpu, c, H, new, window=window, seed=12, behind=1)
        check_attention(o, l, ref, window)


def test_more_new_tokens_than_the_bound_says(gpu):
    # p->chunk only chooses the kernel: sequences with more new tokens are computed all the same
    new = [40, 3, 90]
    for dtype in (BF, F32):
        c = Cache(dtype, 2, 128, 16, [100, 3, 91], seed=2)
        o, l, ref = run(gpu, c, 8, new, seed=2, chunk=1)
        ref = attention(c, *_again(c, new, 2), 0, float(np.float32(1 / math.sqrt(128))), [dtype == BF] * 3)
        check_attention(o, l, ref, dtype)


def _again(c, new, seed):
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    return W.store(rng.standard_normal((sum(new), 8, c.D), dtype=np.float32), c.dtype), new


def test_many_short_sequences(gpu):
    rng = np.random.Generator(np.random.PCG64(4))
    lens = rng.integers(0, 40, size=700).tolist()
    new = [int(rng.integers(0, n + 1)) if i % 3 else 1 for i, n in enumerate(lens)]
    for dtype in (BF, F32):
        c = Cache(dtype, 1, 64, 8, lens, seed=4)
        o, l, ref = run(gpu, c, 4, new, seed=4)
        check_attention(o, l, ref, dtype)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1], [200, 5]])
def test_the_same_call_gives_the_same_bits_and_lse_may_be_left_out(gpu, dtype, new):
    from paper_2411_02886_amd.runtime import to_device
    c = Cache(dtype, 2, 128, 16, [5000, 3001], seed=6)
    p, _, _ = c.problem(8, chunk=max(new))
    T = sum(new)
    q = to_device(W.store(np.random.default_rng(0).standard_normal((T, 8, 128), dtype=np.float32), dtype))
    ind = to_device(np.cumsum([0] + new).astype(np.int32))
    ws = workspace(gpu, p, T)
    outs = []
    for i in range(3):
        out, lse = torch.zeros_like(q), torch.zeros((T, 8), device="cuda:0")
        gpu.ts_paged_attn(p, q, ind, T, 0, 0.09, out, lse if i < 2 else None, ws)
        ws.fill_(-1)
        outs.append((out, lse))
    torch.cuda.synchronize()
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1]) and torch.equal(outs[0][0], outs[2][0])
    assert not outs[2][1].any()


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 1, 1], [130, 1, 3]])
def test_two_streams_and_graphs(gpu, dtype, new):
    """Two calls at once on workspaces of their own; a captured call replayed with eager work and other lengths between."""
    from paper_2411_02886_amd.runtime import to_device
    c = Cache(dtype, 2, 64, 16, [4000, 900, 2500], seed=8)
    p, _, _ = c.problem(8, chunk=max(new))
    T = sum(new)
    ind = to_device(np.cumsum([0] + new).astype(np.int32))
    rng = np.random.default_rng(1)
    q = [to_device(W.store(rng.standard_normal((T, 8, 64), dtype=np.float32), dtype)) for _ in range(2)]
    ref = []
    ws = [workspace(gpu, p, T) for _ in range(2)]

    def call(i, out, lse):
        gpu.ts_paged_attn(p, q[i], ind, T, 0, 0.125, out, lse, ws[i])

    for i in range(2):
        ref.append((torch.zeros_like(q[0]), torch.zeros((T, 8), device="cuda:0")))
        call(i, *ref[i])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = [(torch.zeros_like(q[0]), torch.zeros((T, 8), device="cuda:0")) for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(4):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                call(i, *got[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert torch.equal(got[i][0], ref[i][0]) and torch.equal(got[i][1], ref[i][1])
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=streams[0]):
        call(0, *got[0])
    lens = p._keep[4]
    for rep in range(4):
        for t in got[0]:
            t.zero_()
        if rep == 2:                                     # the lengths are read when the graph runs
            lens -= 130
            call(1, *got[1])
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        if rep < 2:
            assert torch.equal(got[0][0], ref[0][0]) and torch.equal(got[0][1], ref[0][1])
        else:
            want = (torch.zeros_like(q[0]), torch.zeros((T, 8), device="cuda:0"))
            call(0, *want)
            torch.cuda.synchronize()
            assert torch.equal(got[0][0], want[0]) and torch.equal(got[0][1], want[1])
            assert not torch.equal(got[0][1], ref[0][1])


def test_a_pool_beyond_32_bits(gpu):
    """Rows whose byte offset passes 2^32: the last pages of a pool of 5 GiB."""
    P, H_kv, D, H, n = 16, 8, 128, 32, 700
    pages = (5 << 30) // (P * H_kv * D * 2)
    k = torch.zeros((pages, P, H_kv, D), dtype=torch.int16, device="cuda:0")
    v = torch.zeros_like(k)
    small = Cache(BF, H_kv, D, P, [n], seed=3, spare=0)
    from paper_2411_02886_amd.runtime import to_device, to_host
    k[pages - small.pages.size:] = to_device(small.k_bits.reshape(-1, P, H_kv, D))
    v[pages - small.pages.size:] = to_device(small.v_bits.reshape(-1, P, H_kv, D))
    sm = 1 / math.sqrt(D)
    for chunk in (1, 100):
        p = gpu.Problem(batch=1, chunk=chunk, num_q_heads=H, num_kv_heads=H_kv, head_dim=D, page_size=P, max_seq_len=n, dtype=BF,
                        k_pool=k, v_pool=v, page_indptr=to_device(small.indptr),
                        page_indices=to_device((small.pages + pages - small.pages.size).astype(np.int32)), seq_lens=to_device(small.lens))
        q = W.store(np.random.default_rng(2).standard_normal((chunk, H, D), dtype=np.float32), BF)
        out = torch.zeros((chunk, H, D), dtype=torch.int16, device="cuda:0")
        lse = torch.zeros((chunk, H), device="cuda:0")
        gpu.ts_paged_attn(p, to_device(q), None, chunk, 0, sm, out, lse, workspace(gpu, p, chunk))
        torch.cuda.synchronize()
        ref = attention(small, q, [chunk], 0, float(np.float32(sm)), [chunk * 4 > 32])
        check_attention(W.as_f32(to_host(out, bits16=True), BF).astype(np.float64), to_host(lse).astype(np.float64), ref, chunk)


LOOSE = 1 << 20      # a bound far above the lengths: tiles are cut into shares however short they are


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS + [(128, 16), (96, 32)])
def test_shares_of_every_head_layout(gpu, dtype, D, H, H_kv):
    new, old = [65, 1, 0, 70, 3], [700, 900, 5, 131, 0]
    c = Cache(dtype, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H * 19 + D)
    o, l, ref = run(gpu, c, H, new, seed=H, max_seq_len=LOOSE)
    check_attention(o, l, ref, "prompts")
    o, l, ref = run(gpu, c, H, [1] * 5, packed=False, seed=H, max_seq_len=LOOSE)
    check_attention(o, l, ref, "tokens")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("window", [1, 63, 100, 1000])
@pytest.mark.parametrize("D", [64, 128])
def test_windows_in_shares(gpu, dtype, window, D):
    new = [1, 90, 0, 5, 600, 1]
    c = Cache(dtype, 2, D, 8, [3000, 290, 17, 5, 1517, 2], seed=window)
    o, l, ref = run(gpu, c, 6, new, window=window, seed=3, max_seq_len=LOOSE)
    check_attention(o, l, ref, window)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 2, 33, 63, 64, 65, 256, 257, 600])
@pytest.mark.parametrize("loose", [False, True], ids=["", "loose bound"])
def test_batches(gpu, dtype, B, loose):
    rng = np.random.Generator(np.random.PCG64(B))
    lens = rng.integers(0, 300, size=B).tolist()
    c = Cache(dtype, 2, 64, 16, lens, seed=B)
    bound = LOOSE if loose else None
    o, l, ref = run(gpu, c, 8, [1] * B, packed=False, seed=B, max_seq_len=bound)
    check_attention(o, l, ref, "tokens")
    new = [min(n, int(rng.integers(0, 3) ** 6)) for n in lens]                   # 0, 1 or up to 64
    o, l, ref = run(gpu, c, 8, new, seed=B, max_seq_len=bound, chunk=64)
    check_attention(o, l, ref, "mixed")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 130])
@pytest.mark.parametrize("rise", [400.0, -400.0, 60.0])
def test_logits_that_rise_or_fall_along_the_sequence(gpu, dtype, D, n, rise):
    """From 0 to `rise` over 3000 tokens: far beyond what the first tiles' largest logit says, or far below it."""
    N = 3000
    c = Cache(dtype, 2, D, 16, [N, N - 900], seed=n)
    for b in range(2):
        at = c.slots(b)
        t = np.arange(len(at)) / N
        k = 0.1 * c.k[at] + (rise * t * math.sqrt(D) / D)[:, None, None]        # queries are near 1 in every element
        bits = W.store(k.astype(np.float32), dtype)
        c.k_bits[at], c.k[at] = bits, W.as_f32(bits, dtype).astype(np.float64)
    rng = np.random.Generator(np.random.PCG64(5))
    q = W.store((1 + 0.1 * rng.standard_normal((2 * n, 8, D))).astype(np.float32), dtype)
    from paper_2411_02886_amd.runtime import to_device, to_host
    for bound in (None, LOOSE):
        p, _, _ = c.problem(8, chunk=n, max_seq_len=bound)
        out = torch.zeros((2 * n, 8, D), dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0")
        lse = torch.zeros((2 * n, 8), device="cuda:0")
        gpu.ts_paged_attn(p, to_device(q), None, 2 * n, 0, 1 / math.sqrt(D), out, lse, workspace(gpu, p, 2 * n))
        torch.cuda.synchronize()
        ref = attention(c, q, [n, n], 0, float(np.float32(1 / math.sqrt(D))), [dtype == BF and n * 4 > 32] * 2)
        check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64), ref, bound)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("n", [1, 100])
def test_a_broken_sequence_leaves_the_others_alone(gpu, dtype, bad, n):
    """Its own rows are unspecified; the call ends, and the other sequences' bits do not change."""
    from paper_2411_02886_amd.runtime import to_device
    lens = [900, 700, 333]
    c = Cache(dtype, 2, 64, 16, lens, seed=4)
    rng = np.random.Generator(np.random.PCG64(5))
    q = to_device(W.store(rng.standard_normal((3 * n, 8, 64), dtype=np.float32), dtype))
    got = []
    for broken in (False, True):
        p, k, v = c.problem(8, chunk=n, max_seq_len=LOOSE)
        if broken:
            at = torch.tensor(c.slots(1)[::7], device="cuda:0")
            val = torch.tensor([bad]).to(torch.bfloat16).view(torch.int16)[0] if dtype == BF else torch.tensor(bad)
            for x in (k, v):
                x.view(-1, 2, 64)[at] = val.to("cuda:0")
        out, lse = torch.zeros_like(q), torch.zeros((3 * n, 8), device="cuda:0")
        gpu.ts_paged_attn(p, q, None, 3 * n, 0, 0.125, out, lse, workspace(gpu, p, 3 * n))
        torch.cuda.synchronize()
        got.append((out, lse))
    for rows in (slice(0, n), slice(2 * n, 3 * n)):
        assert torch.equal(got[0][0][rows], got[1][0][rows]) and torch.equal(got[0][1][rows], got[1][1][rows])


def test_more_new_tokens_than_the_bound_says_in_shares(gpu):
    new = [40, 3, 90]
    for dtype in (BF, F32):
        for H in (8, 4):
            c = Cache(dtype, 2, 128, 16, [400, 3, 291], seed=2)
            o, l, _ = run(gpu, c, H, new, seed=2, chunk=1, max_seq_len=LOOSE)
            rng = np.random.Generator(np.random.PCG64(1002))
            q = W.store(rng.standard_normal((sum(new), H, 128), dtype=np.float32), dtype)
            ref = attention(c, q, new, 0, float(np.float32(1 / math.sqrt(128))), [dtype == BF] * 3)
            check_attention(o, l, ref, dtype)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,D", [(8, 64), (4, 128)])
@pytest.mark.parametrize("window", [1, 20, 100, 300])
def test_tokens_in_front_of_every_window_are_not_read(gpu, dtype, H, D, window):
    new, lens = [1, 4, 13, 150], [900, 333, 517, 800]
    c = Cache(dtype, 2, D, 16, lens, seed=window)
    nan = 0x7fc0 if dtype == BF else np.nan
    for b, (n, N) in enumerate(zip(new, lens)):
        first = max(0, N - n - window + 1)
        at = c.slots(b)[:first]
        c.k_bits[at], c.v_bits[at] = nan, nan
        c.pages[c.indptr[b]:c.indptr[b] + first // 16] = c.spare[0]            # pages of full NaN stand for those that are gone
    for bound in (None, LOOSE):
        o, l, ref = run(gpu, c, H, new, window=window, seed=9, max_seq_len=bound)
        check_attention(o, l, ref, (window, bound))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("H,H_kv,D", [(32, 8, 128), (32, 8, 64), (28, 4, 128), (16, 16, 64), (24, 8, 128)])
@pytest.mark.parametrize("window", [0, 77])
def test_prompts_of_many_whole_tiles(gpu, dtype, H, H_kv, D, window):
    """More than 512 tiles of 32 rows and no more than 256 large ones, up to 1024 keys: a workgroup per large tile."""
    new, old = [421, 5, 300, 1, 64, 500], [200, 900, 0, 17, 0, 1]
    c = Cache(dtype, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H + D)
    o, l, ref = run(gpu, c, H, new, window=window, seed=21, behind=2)
    check_attention(o, l, ref, window)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("sm", [0.0, -0.3, 40.0])
def test_scales_in_whole_large_tiles(gpu, dtype, sm):
    new = [640, 260]
    c = Cache(dtype, 8, 64, 16, [700, 270], seed=8)
    o, l, ref = run(gpu, c, 32, new, sm=sm, seed=8)
    check_attention(o, l, ref, sm)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("B", [1, 63, 64, 65, 4096, 4097])
def test_packed_batches_of_short_sequences(gpu, dtype, B):
    """A search among 64 places at a time: one, two and three steps; sequences without new tokens between the others."""
    new = [(0, 1, 3, 1, 17)[b % 5] if b % 64 < 60 else 0 for b in range(B)]
    lens = [(n + b % 7) % 30 for b, n in enumerate(new)]
    c = Cache(dtype, 2, 64, 4, lens, seed=B)
    o, l, ref = run(gpu, c, 4, new, seed=B, behind=3)
    check_attention(o, l, ref, B)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("bad", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("H,D", [(8, 64), (4, 128)])
def test_keys_that_a_row_does_not_see_may_be_anything(gpu, dtype, bad, H, D):
    """The last new token of each sequence has a broken key: the rows before it do not see it (its own are unspecified)."""
    new, lens = [2, 9, 130, 40], [700, 9, 333, 1000]
    c = Cache(dtype, 2, D, 16, lens, seed=6)
    bits = {np.nan: 0x7fc0, np.inf: 0x7f80, -np.inf: 0xff80}[bad] if dtype == BF else bad
    at = [int(c.slots(b)[-1]) for b in range(4)]
    c.k_bits[at] = bits
    last = np.cumsum(new) - 1
    rows = np.setdiff1d(np.arange(sum(new)), last)
    for bound in (None, LOOSE):
        o, l, ref = run(gpu, c, H, new, seed=10, max_seq_len=bound)           # (c.k, which the reference reads, is whole)
        check_attention(o[rows], l[rows], tuple(x[rows] for x in ref), (bad, bound))
