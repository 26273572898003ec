"""ts_quant_attn against the definition in 64 bits, of what the codes and scales stand for: lengths from nothing to thousands, packed and padded rows,
windows, trees, page sizes, head layouts, rows that see nothing, neighbours full of NaN, scales that are no number, graphs and streams."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import check_attention
from quant_util import QuantPages
from tree_util import attention, closure, random_tree, words_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
CODES = pytest.mark.parametrize("code", [0, 1], ids=["int8", "e4m3"])


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


def run(ts, c, H, new, window=0, packed=True, sm=None, seed=0, max_seq_len=None, q_scale=1.0, behind=0, chunk=None, sees=None, words=None):
    from paper_2411_02886_amd.runtime import to_host
    D, T = c.D, sum(new) + behind
    sm = 1.0 / math.sqrt(D) if sm is None else sm
    rng = np.random.Generator(np.random.PCG64(1000 + seed))
    q = W.store(q_scale * rng.standard_normal((T, H, D), dtype=np.float32), c.dtype)
    p, quant = c.problem(H, chunk=max(1, max(new)) if chunk is None else chunk, max_seq_len=max_seq_len)
    mask = None
    if sees is not None:
        words = max(1, (max(new) + 31) // 32) if words is None else words
        mask = dev(np.concatenate([words_of(s, words) for s in sees if len(s)] + [np.zeros((behind, words), np.uint32)]).view(np.int32))
        sees = [s & (np.arange(len(s)) < 32 * words) for s in sees]
    out = torch.full((T, H, D), 77, dtype=torch.int16 if c.dtype == BF else torch.float32, device="cuda:0")
    lse = torch.full((T, H), 55.0, dtype=torch.float32, device="cuda:0")
    n = ts.ts_quant_attn_workspace_bytes(p, T)
    ws = torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")       # NaN in every word: nothing may be read first
    ts.ts_quant_attn(p, quant, dev(q), dev(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None, T, window, mask, sm, out, lse, ws)
    torch.cuda.synchronize()
    o, l = to_host(out, bits16=c.dtype == BF), to_host(lse)
    if behind:
        assert np.all(o[T - behind:] == 77) and np.all(l[T - behind:] == 55.0)
    # More roundings: the key's scale times the call's, and the product with it; the weight times the value's scale.  Tiny: a key's weight times its scale, and each of the
    # three parts of that, is 0 where it would be below the smallest normal number, 2^-126.  It multiplies codes of up to 448, and the row's sum of weights is at least 2^-7
    # (the reference lies at most 6 above the largest exponent, plus rounding): at most 4 * 2^-126 * 2^9 * 2^7 = 2^-108.  Codes may be exactly 0, so that an output can be so small.
    ref = attention(c, q[:T - behind], new, window, float(np.float32(sm)), sees, more=4, tiny=2.0 ** -108)
    return W.as_f32(o, c.dtype).astype(np.float64)[:T - behind], l[:T - behind].astype(np.float64), ref


def trees(new, seed, **kw):
    rng = np.random.default_rng(seed)
    return [closure(random_tree(rng, n, **kw)) for n in new]


HEADS = [(1, 1), (8, 8), (8, 4), (6, 2), (8, 2), (10, 2), (6, 1), (28, 4), (16, 2), (32, 32)]


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_single_tokens_of_every_head_layout(gpu, dtype, code, D, H, H_kv):
    lens = [1, 2, 15, 16, 17, 127, 128, 129, 300, 1]
    c = QuantPages(dtype, code, H_kv, D, 16, lens, seed=H * 131 + D)
    check_attention(*run(gpu, c, H, [1] * len(lens), packed=False, seed=H), "tokens")


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
def test_prompts_of_every_head_layout(gpu, dtype, code, D, H, H_kv):
    new, old = [65, 1, 70], [0, 40, 131]
    c = QuantPages(dtype, code, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H * 17 + D)
    check_attention(*run(gpu, c, H, new, seed=H), "prompts")


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 2, 3, 7, 8, 9, 15, 16, 17, 31, 33, 63, 64, 65, 100, 129, 257])
def test_lengths_of_a_chunk(gpu, dtype, code, D, n):
    c = QuantPages(dtype, code, 2, D, 16, [n, n + 1, n + 63, n + 64, n + 200], seed=n)
    check_attention(*run(gpu, c, 8, [n] * 5, packed=False, seed=n), n)


@DTYPES
@CODES
@pytest.mark.parametrize("window", [1, 2, 15, 31, 32, 33, 100, 128, 1 << 30])
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_windows(gpu, dtype, code, window, tree):
    new = [1, 90, 0, 5, 200]
    c = QuantPages(dtype, code, 2, 64 if window % 2 else 128, 8, [300, 290, 17, 5, 517], seed=window % 1000)
    check_attention(*run(gpu, c, 6, new, window=window, seed=3, sees=trees(new, window % 97) if tree else None), window)


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 5, 31, 32, 33, 64, 65, 130])
def test_trees(gpu, dtype, code, D, n):
    new, old = [n, 1, max(1, n // 2), 0], [200, 31, 0, 7]
    c = QuantPages(dtype, code, 2, D, 16, [a + b for a, b in zip(new, old)], seed=n)
    check_attention(*run(gpu, c, 8, new, seed=n, sees=trees(new, n, roots=True)), n)
    rng = np.random.default_rng(n)
    sees = [rng.random((m, m)) < 0.3 for m in new]
    sees[0][n // 2] = False
    check_attention(*run(gpu, c, 8, new, seed=n, sees=sees, words=1), "any bits")


@DTYPES
@CODES
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
def test_sequences_without_tokens_and_rows_that_see_nothing(gpu, dtype, code, tree):
    new, lens = [0, 3, 70, 2, 0, 1, 40], [0, 0, 30, 2, 9, 0, 41]
    c = QuantPages(dtype, code, 4, 64, 16, lens, seed=5)
    check_attention(*run(gpu, c, 8, new, seed=5, behind=3, sees=trees(new, 1) if tree else None), "empty")


@DTYPES
@CODES
@pytest.mark.parametrize("P", [1, 4, 8, 32, 64, 256])
@pytest.mark.parametrize("chunk", [1, 50])
def test_page_sizes(gpu, dtype, code, P, chunk):
    c = QuantPages(dtype, code, 2, 128, P, [chunk + 333, chunk + 64], seed=P)
    check_attention(*run(gpu, c, 8, [chunk] * 2, packed=False, seed=P), P)


@DTYPES
@CODES
@pytest.mark.parametrize("sm,q_scale", [(0.0, 1.0), (-0.3, 1.0), (1.0, 4.0), (64.0, 30.0)])
@pytest.mark.parametrize("n", [1, 60])
def test_scales_and_large_logits(gpu, dtype, code, sm, q_scale, n):
    c = QuantPages(dtype, code, 2, 64, 16, [n + 150, n + 40], seed=n, scale=q_scale)
    check_attention(*run(gpu, c, 8, [n] * 2, packed=False, sm=sm, q_scale=q_scale, seed=n), (sm, q_scale))


@pytest.mark.parametrize("dtype,H,H_kv,D,new,old", [(BF, 32, 8, 128, [1] * 5, [9000, 3, 20001, 128, 5000]), (F32, 8, 2, 64, [1] * 3, [6000, 1, 11000]),
                                                    (BF, 4, 4, 64, [1], [12345]), (F32, 16, 4, 128, [1, 9], [5001, 70]), (BF, 28, 4, 128, [70, 1, 3], [9000, 4000, 1]),
                                                    (F32, 28, 4, 128, [20], [7000])])
@CODES
@pytest.mark.parametrize("loose", [False, True], ids=["", "loose bound"])
def test_long_caches_are_cut_into_shares(gpu, dtype, H, H_kv, D, new, old, code, loose):
    c = QuantPages(dtype, code, H_kv, D, 16, [a + b for a, b in zip(new, old)], seed=H)
    check_attention(*run(gpu, c, H, new, seed=H, max_seq_len=300000 if loose else None, chunk=40 if loose else None), old)


# A bound that promises long sequences gives a workgroup several KV heads at once; what the sequences have is another matter.
@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", HEADS)
@pytest.mark.parametrize("new", [[1] * 5, [2, 1, 0, 9, 4]], ids=["tokens", "drafts"])
def test_heads_side_by_side(gpu, dtype, code, D, H, H_kv, new):
    c = QuantPages(dtype, code, H_kv, D, 16, [1, 300, 33, 2500, 700], seed=H + D)
    check_attention(*run(gpu, c, H, new, max_seq_len=1 << 24, seed=H), (H, H_kv))


@DTYPES
@CODES
@pytest.mark.parametrize("H,H_kv", [(8, 8), (6, 2), (28, 4), (4, 1)])
@pytest.mark.parametrize("window", [0, 1 << 23])
def test_trees_with_heads_side_by_side(gpu, dtype, code, H, H_kv, window):
    new = [13, 1, 70, 5, 0, 33]
    c = QuantPages(dtype, code, H_kv, 64, 16, [13, 400, 2000, 90, 11, 20], seed=H)     # the last has fewer tokens than new ones: rows that see nothing
    check_attention(*run(gpu, c, H, new, window=window, max_seq_len=1 << 24, sees=trees(new, H), seed=H, behind=3), (H, H_kv))


def test_many_sequences(gpu):
    rng = np.random.Generator(np.random.PCG64(4))
    lens = rng.integers(0, 60, size=700).tolist()
    new = [int(rng.integers(0, min(n, 20) + 1)) for n in lens]
    c = QuantPages(BF, 0, 1, 64, 8, lens, seed=6)
    check_attention(*run(gpu, c, 4, new, seed=6), "many")
    check_attention(*run(gpu, c, 4, new, seed=6, sees=trees(new, 6)), "many trees")


@DTYPES
@CODES
@pytest.mark.parametrize("n", [1, 40])
def test_a_scale_that_is_no_number_concerns_the_rows_that_see_it(gpu, dtype, code, n):
    """Rows of K or V that held an infinity or a NaN: NaN for the rows that see them, nothing for those that do not."""
    H_kv, D, old = 2, 64, 100
    for name in "kv":
        c = QuantPages(dtype, code, H_kv, D, 16, [n + old, n + old], seed=n)
        s = c.slots(0)[old + n - 1]                          # the last token: only the last row sees it
        c.scales[name][s] = np.nan
        for x in (c.k if name == "k" else c.v,):
            x[s] = np.nan
        o, l, ref = run(gpu, c, 8, [n, n], seed=n)
        rest = np.arange(2 * n) != n - 1
        assert np.isnan(o[n - 1]).all() and (name == "v" or np.isnan(l[n - 1]).all())
        check_attention(o[rest], l[rest], [x[rest] for x in ref], name)


@CODES
def test_a_captured_call_reads_lengths_when_it_runs_and_two_streams_run_at_once(gpu, code):
    c = QuantPages(BF, code, 2, 64, 16, [3000, 40, 700], seed=1)
    p, quant = c.problem(8, chunk=4)
    rng = np.random.default_rng(0)
    q = [dev(W.store(rng.standard_normal((12, 8, 64), dtype=np.float32), BF)) for _ in range(2)]
    mask = dev(words_of(np.tril(np.ones((4, 4), bool)), 1).view(np.int32)).repeat(3, 1)
    ws = [torch.empty((gpu.ts_quant_attn_workspace_bytes(p, 12) // 4,), dtype=torch.int32, device="cuda:0") for _ in range(2)]
    out = [torch.zeros_like(x) for x in q]
    lse = [torch.zeros((12, 8), device="cuda:0") for _ in range(2)]

    def call(i, o, l):
        gpu.ts_quant_attn(p, quant, q[i], None, 12, 0, mask if i else None, 0.125, o, l, ws[i])

    streams = [torch.cuda.Stream() for _ in range(2)]
    graphs = []
    torch.cuda.synchronize()
    for i in range(2):
        with torch.cuda.stream(streams[i]):
            call(i, out[i], lse[i])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=streams[i]):
            call(i, out[i], lse[i])
    for rep in range(4):
        for x in (*out, *lse):
            x.zero_()
        torch.cuda.synchronize()
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                graphs[i].replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (*out, *lse)]
        for i in range(2):
            call(i, out[i], lse[i])
        torch.cuda.synchronize()
        for a, b in zip(got, (*out, *lse)):
            assert torch.equal(a, b), rep
        assert torch.equal(got[0], got[1]) == torch.equal(q[0], q[1])
        p._keep[4].sub_(5)


def test_nothing_to_do(gpu):
    c = QuantPages(BF, 0, 2, 64, 16, [5], seed=1)
    p, quant = c.problem(8)
    gpu.ts_quant_attn(p, quant, None, None, 0, 0, None, 0.1, None, None, None)
    torch.cuda.synchronize()
