"""The weights of dense attention: ts_paged_attn keeps them in float whatever the rows, ts_paged_attn_rounded may round bf16 ones."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache, attention, check_attention

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
LOOSE = 1 << 20      # a bound far above the lengths: tiles are cut into shares however short they are


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def call(ts, c, H, new, rounded=False, window=0, packed=True, bound=None, seed=0, sm=None, q=None):
    """(out, lse, q, scale)"""
    from paper_2411_02886_amd.runtime import to_device, to_host
    D, T = c.D, sum(new)
    sm = 1.0 / math.sqrt(D) if sm is None else sm
    if q is None:
        q = W.store(np.random.Generator(np.random.PCG64(seed)).standard_normal((T, H, D), dtype=np.float32), c.dtype)
    p, _, _ = c.problem(H, chunk=max(1, max(new)), max_seq_len=bound)
    ind = to_device(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None
    n = ts.ts_paged_attn_workspace_bytes(p, T)
    ws = torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")
    out = torch.full((T, H, D), 77, dtype=torch.int16 if c.dtype == BF else torch.float32, device="cuda:0")
    lse = torch.full((T, H), 55.0, dtype=torch.float32, device="cuda:0")
    (ts.ts_paged_attn_rounded if rounded else ts.ts_paged_attn)(p, to_device(q), ind, T, window, sm, out, lse, ws)
    torch.cuda.synchronize()
    return W.as_f32(to_host(out, bits16=c.dtype == BF), c.dtype).astype(np.float64), to_host(lse).astype(np.float64), q, float(np.float32(sm))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", [(8, 2), (28, 4), (6, 2), (8, 8), (16, 2)])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
def test_bf16_weights_are_not_rounded(gpu, D, H, H_kv, window, bound):
    """The bounds of float weights hold for prompts and chunks of every length."""
    new, old = [130, 1, 300, 17, 0, 64], [900, 40, 0, 131, 5, 2000]
    c = Cache(BF, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H + D)
    out, lse, q, sm = call(gpu, c, H, new, window=window, bound=bound)
    check_attention(out, lse, attention(c, q, new, window, sm, [False] * len(new)), (H, window))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [33, 65, 129, 500, 1025])
def test_bf16_weights_of_padded_prompts_are_not_rounded(gpu, D, n):
    for old in (0, 77, 1500):
        c = Cache(BF, 2, D, 16, [n + old] * 2, seed=n)
        out, lse, q, sm = call(gpu, c, 8, [n] * 2, packed=False)
        check_attention(out, lse, attention(c, q, [n] * 2, 0, sm, [False] * 2), (n, old))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 100])
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
def test_rounded_weights(gpu, D, window, bound):
    new, old = [130, 1, 300, 17, 0, 64], [900, 40, 0, 131, 5, 2000]
    for dtype in (BF, F32):
        c = Cache(dtype, 2, D, 16, [a + b for a, b in zip(new, old)], seed=D)
        out, lse, q, sm = call(gpu, c, 8, new, rounded=True, window=window, bound=bound)
        check_attention(out, lse, attention(c, q, new, window, sm, [dtype == BF and n * 4 > 32 for n in new]), (dtype, window))


@pytest.mark.parametrize("rise", [400.0, -400.0, 60.0])
@pytest.mark.parametrize("sm", [None, -0.2])
@pytest.mark.parametrize("D", [64, 128])
def test_rising_and_falling_logits(gpu, rise, sm, D):
    """The reference is fixed by the first tiles; a piece whose logits leave it far below is done again."""
    n, N = 130, 3000
    c = Cache(BF, 2, D, 16, [N, N - 900], seed=1)
    for b in range(2):
        at = c.slots(b)
        k = 0.1 * c.k[at] + (rise * np.arange(len(at)) / N * math.sqrt(D) / D)[:, None, None]
        c.k_bits[at] = W.store(k.astype(np.float32), BF)
        c.k[at] = W.as_f32(c.k_bits[at], BF)
    q = W.store((1 + 0.1 * np.random.default_rng(5).standard_normal((2 * n, 8, D))).astype(np.float32), BF)
    for rounded in (False, True):
        for bound in (None, LOOSE):
            out, lse, _, scale = call(gpu, c, 8, [n, n], rounded=rounded, packed=False, bound=bound, sm=sm, q=q)
            check_attention(out, lse, attention(c, q, [n, n], 0, scale, [rounded] * 2), (rounded, bound))


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
def test_an_infinite_value_that_every_row_sees_comes_out_infinite(gpu, D, bound):
    n, N = 200, 1000
    for rounded in (False, True):
        c = Cache(BF, 2, D, 16, [N], seed=2)
        at = c.slots(0)
        c.v_bits[at[10], :, 3], c.v_bits[at[500], :, 40] = 0x7f80, 0xff80
        c.v[at[10], :, 3], c.v[at[500], :, 40] = 0.0, 0.0          # (what the reference reads; these two columns are looked at by themselves)
        out, lse, q, sm = call(gpu, c, 8, [n], rounded=rounded, bound=bound)
        assert np.all(out[..., 3] == np.inf) and np.all(out[..., 40] == -np.inf)
        ref = attention(c, q, [n], 0, sm, [rounded])
        out[..., [3, 40]] = ref[0][..., [3, 40]]
        check_attention(out, lse, ref, bound)


def test_both_forms_agree_where_nothing_is_rounded(gpu):
    """fp32, and bf16 sequences of up to 32 rows: the same bits."""
    for dtype, new in ((F32, [1, 90, 300]), (BF, [1, 8, 3])):
        c = Cache(dtype, 2, 64, 16, [900, 700, 333], seed=4)
        a, b = call(gpu, c, 8, new), call(gpu, c, 8, new, rounded=True)
        assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("rounded", [False, True])
def test_graph_of_a_prompt(gpu, rounded):
    from paper_2411_02886_amd.runtime import to_device
    c = Cache(BF, 2, 128, 16, [1500, 300], seed=7)
    new = [400, 290]
    p, _, _ = c.problem(8, chunk=400)
    ind = to_device(np.cumsum([0] + new).astype(np.int32))
    q = to_device(W.store(np.random.default_rng(0).standard_normal((690, 8, 128), dtype=np.float32), BF))
    ws = torch.empty((gpu.ts_paged_attn_workspace_bytes(p, 690) + 255) // 256 * 64, dtype=torch.int32, device="cuda:0")
    out, lse = torch.zeros_like(q), torch.zeros((690, 8), device="cuda:0")
    attend = gpu.ts_paged_attn_rounded if rounded else gpu.ts_paged_attn
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        attend(p, q, ind, 690, 0, 0.09, out, lse, ws)
    torch.cuda.synchronize()
    want = out.clone(), lse.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        attend(p, q, ind, 690, 0, 0.09, out, lse, ws)
    for rep in range(3):
        out.zero_(), lse.zero_(), ws.fill_(-1)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[0]) and torch.equal(lse, want[1]), rep


@pytest.mark.parametrize("rounded", [False, True])
def test_attend_all_takes_the_choice(gpu, rounded):
    from paper_2411_02886_amd.runtime import ChunkSelector, to_device, to_host
    C = 100
    c = Cache(BF, 2, 64, 16, [700], seed=9)
    sel = ChunkSelector(C=C, H=8, H_kv=2, D=64, P=16, k=16, k_pool=c.k_bits.reshape(-1, 16, 2, 64), v_pool=c.v_bits.reshape(-1, 16, 2, 64),
                        page_indptr=c.indptr, page_indices=c.pages, seq_lens=c.lens)
    q = W.store(np.random.default_rng(3).standard_normal((C, 8, 64), dtype=np.float32), BF)
    sel.attend_all(to_device(q), round_weights=rounded)
    torch.cuda.synchronize()
    out, lse = W.as_f32(to_host(sel.out, bits16=True), BF).astype(np.float64).reshape(C, 8, 64), to_host(sel.lse).astype(np.float64).reshape(C, 8)
    check_attention(out, lse, attention(c, q, [C], 0, 0.125, [rounded]), rounded)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 300])
@pytest.mark.parametrize("D", [64, 128])
def test_large_values_beside_rising_logits_stay_finite(gpu, dtype, n, D):
    """Logits rise by 40 along the sequence, values are around 2^100: a weight of 2^50 times one of them is no float, the result is.  (300 tokens
    times 32 heads: large tiles, a workgroup's each.)"""
    N, H, H_kv = 700, 32, 8
    c = Cache(dtype, H_kv, D, 16, [N, N - 50], seed=1)
    for b in range(2):
        at = c.slots(b)
        k = 0.1 * c.k[at] + (40.0 * np.arange(len(at)) / N * math.sqrt(D) / D)[:, None, None]
        c.k_bits[at] = W.store(k.astype(np.float32), dtype)
        c.v_bits[at] = W.store((2.0 ** 100 * c.v[at]).astype(np.float32), dtype)
        c.k[at], c.v[at] = W.as_f32(c.k_bits[at], dtype), W.as_f32(c.v_bits[at], dtype)
    q = W.store((1 + 0.1 * np.random.default_rng(5).standard_normal((2 * n, H, D))).astype(np.float32), dtype)
    for rounded in (False, True):
        for bound in (None, LOOSE):
            out, lse, _, scale = call(gpu, c, H, [n, n], rounded=rounded, packed=False, bound=bound, q=q)
            assert np.isfinite(out).all(), (rounded, bound)
            check_attention(out, lse, attention(c, q, [n, n], 0, scale, [rounded and dtype == BF and n * 4 > 32] * 2), (rounded, bound))


@pytest.mark.parametrize("rounded", [False, True], ids=["", "rounded"])
@pytest.mark.parametrize("n", [3, 12, 24, 30, 50])
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
def test_full_packed_batches_are_computed_as_padded_ones(gpu, rounded, n, bound):
    """The same rows, described by q_indptr or by the chunk: the same kernel, the same bits."""
    c = Cache(BF, 2, 64, 16, [3000, 2000, 1500, 700], seed=n)
    a, b = (call(gpu, c, 8, [n] * 4, rounded=rounded, packed=packed, bound=bound) for packed in (True, False))
    assert np.array_equal(a[0], b[0]) and np.array_equal(a[1], b[1])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("longest", [900, 1024, 1025, 1500, 2100])
@pytest.mark.parametrize("rounded", [False, True], ids=["", "rounded"])
def test_single_tokens_beside_a_prompt(gpu, dtype, longest, rounded):
    """Sequences with few rows by a workgroup each or in shares, beside large tiles."""
    new, lens = [1, 200, 1, 2, 0, 1], [longest, 200, 3, longest - 7, 50, 1]
    c = Cache(dtype, 2, 64, 16, lens, seed=longest)
    out, lse, q, sm = call(gpu, c, 8, new, rounded=rounded)
    check_attention(out, lse, attention(c, q, new, 0, sm, [rounded and dtype == BF and n * 4 > 32 for n in new]), longest)
