"""Masks among the new tokens beside what they stand for: the lower triangle is the causal call, in captured graphs too, and a key that holds infinities is
no number to the row that sees it and nothing to the others."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache, check_attention
from quant_util import QuantPages
from tree_util import attention, words_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])


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


@DTYPES
@pytest.mark.parametrize("code", [0, 1], ids=["int8", "e4m3"])
@pytest.mark.parametrize("n", [4, 40])
def test_replays_of_the_causal_call_and_of_the_lower_triangle(gpu, dtype, code, n):
    """Both captured with the same queries: every replay against the definition, with the lengths that it finds."""
    from paper_2411_02886_amd.runtime import to_host
    H, D, lens = 8, 64, [3000, 90, 700]
    c = QuantPages(dtype, code, 2, D, 16, lens, seed=n)
    p, quant = c.problem(H, chunk=n)
    T, sm = 3 * n, 1 / math.sqrt(D)
    q = W.store(np.random.default_rng(n).standard_normal((T, H, D), dtype=np.float32), dtype)
    triangle, words = np.tril(np.ones((n, n), bool)), (n + 31) // 32
    q_dev, mask = dev(q), dev(np.concatenate([words_of(triangle, words)] * 3).view(np.int32))
    ws = [torch.empty((gpu.ts_quant_attn_workspace_bytes(p, T) // 4,), dtype=torch.int32, device="cuda:0") for _ in range(2)]
    out = [torch.zeros_like(q_dev) for _ in range(2)]
    lse = [torch.zeros((T, H), device="cuda:0") for _ in range(2)]

    def call(i):
        gpu.ts_quant_attn(p, quant, q_dev, None, T, 0, mask if i else None, sm, out[i], lse[i], ws[i])

    graphs, stream = [], torch.cuda.Stream()
    torch.cuda.synchronize()
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[i], stream=stream):
            call(i)
    for rep in range(3):
        for x in (*out, *lse):
            x.zero_()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        ref = attention(c, q, [n] * 3, 0, float(np.float32(sm)), more=4, tiny=2.0 ** -108)
        for i in range(2):
            check_attention(W.as_f32(to_host(out[i], bits16=dtype == BF), dtype).astype(np.float64), to_host(lse[i]).astype(np.float64), ref, (rep, i))
        p._keep[4].sub_(7)
        c.lens = c.lens - 7


@DTYPES
@pytest.mark.parametrize("n", [6, 60, 100])
@pytest.mark.parametrize("bad", [np.nan, np.inf])
def test_a_key_of_infinities_or_nan(gpu, dtype, n, bad):
    """Its products with a query's elements, of both signs, have no sum: NaN for the row that sees it, in out and lse; every other row as if it were not there."""
    from paper_2411_02886_amd.runtime import to_host
    H, D, old = 8, 64, 90
    c = Cache(dtype, 2, D, 16, [n + old], seed=n)
    sees = np.eye(n, dtype=bool) | (np.arange(n) == 0)
    c.k_bits[c.slots(0)[old + 3]] = 0x7fc0 if dtype == BF and np.isnan(bad) else W.store(np.full((2, D), bad, np.float32), dtype)
    q = W.store(np.random.default_rng(n).standard_normal((n, H, D), dtype=np.float32), dtype)
    q32 = W.as_f32(q, dtype)[3]
    assert (q32 > 0).any(axis=-1).all() and (q32 < 0).any(axis=-1).all()
    p, sm, words = c.problem(H, chunk=n)[0], 1 / math.sqrt(D), (n + 31) // 32
    out, lse = torch.zeros((n, H, D), dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0"), torch.zeros((n, H), device="cuda:0")
    ws = torch.full(((gpu.ts_paged_attn_workspace_bytes(p, n) + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")
    gpu.ts_tree_attn(p, dev(q), None, n, 0, dev(words_of(sees, words).view(np.int32)), sm, out, lse, ws)
    torch.cuda.synchronize()
    o, l = W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64)
    assert np.isnan(o[3]).all() and np.isnan(l[3]).all()
    rest = np.arange(n) != 3
    ref = attention(c, q, [n], 0, float(np.float32(sm)), [sees])
    check_attention(o[rest], l[rest], [x[rest] for x in ref], n)
