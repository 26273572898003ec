"""A value's scale that is no number concerns every row that sees the key, also rows whose weight for it is too small for a float: in every kernel, whether the
key comes before or behind those that outweigh it, alone or in another piece of the cache."""
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


def check(ts, dtype, code, new, old, bad, H=8, H_kv=2, D=64, bound=None, tree=False):
    """bad: per sequence the key whose value has a scale of NaN.  Logits of +-100 and more: the key's weight is 0 beside others that are not."""
    from paper_2411_02886_amd.runtime import to_host
    T, lens = sum(new), [a + b for a, b in zip(new, old)]
    rng = np.random.default_rng(T + len(new))
    c = QuantPages(dtype, code, H_kv, D, 16, lens, seed=T)
    sm = 1 / math.sqrt(D)
    q = rng.standard_normal((T, H, D), dtype=np.float32)
    # queries share a direction (by KV head), the bad key points the other way, every seventh key along with it
    way = rng.standard_normal((H_kv, D))
    way /= np.linalg.norm(way, axis=-1, keepdims=True)
    q = W.store(q + 40.0 * way.repeat(H // H_kv, axis=0).astype(np.float32), dtype)
    from quant_util import encode
    for b, t in enumerate(bad):
        at = c.slots(b)
        for s, sign in [(s, 1.0) for s in at[::7]] + [(at[t], -1.0)]:
            x = W.as_f32(W.store((30.0 * sign * way).astype(np.float32), dtype), dtype)
            c.bytes["k"][s], c.scales["k"][s] = encode(x, code)
        c.scales["v"][at[t]] = np.nan
    c.k, c.v = (c.values(c.bytes[n], c.scales[n]) for n in "kv")
    sees = [closure(random_tree(rng, n)) for n in new] if tree else None
    words = (max(new) + 31) // 32
    mask = dev(np.concatenate([words_of(s, words) for s in sees]).view(np.int32)) if tree else None
    p, quant = c.problem(H, chunk=max(new), max_seq_len=bound)
    out, lse = torch.full((T, H, D), 77, dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0"), torch.full((T, H), 55.0, device="cuda:0")
    n = ts.ts_quant_attn_workspace_bytes(p, T)
    ws = torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")
    ts.ts_quant_attn(p, quant, dev(q), dev(np.cumsum([0] + new).astype(np.int32)), T, 0, mask, sm, out, lse, ws)
    torch.cuda.synchronize()
    o, l = W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64)
    ref = attention(c, q, new, 0, float(np.float32(sm)), sees, more=4, tiny=2.0 ** -108)
    lost = np.isnan(ref[0]).any(axis=(1, 2))
    assert lost.any() and np.isnan(ref[0][lost]).all()
    assert np.isnan(o[lost]).all(), np.flatnonzero(~np.isnan(o).all(axis=(1, 2)) & lost)
    check_attention(np.where(lost[:, None, None], 0.0, o), l, [np.where(lost[:, None, None], 0.0, ref[0]), ref[1], np.where(lost[:, None, None], 1.0, ref[2]), ref[3]], bad)


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("n", [1, 8, 30, 60])            # (bf16: 30 and 60 tokens take the kernel of many rows, 128 and 256 of them)
@pytest.mark.parametrize("t", [3, 96, 290])
def test_cached_keys(gpu, dtype, code, D, n, t):
    check(gpu, dtype, code, [n, n], [300, 291], [t, t], D=D)


@DTYPES
@CODES
@pytest.mark.parametrize("n", [1, 30])
@pytest.mark.parametrize("t", [5, 4000, 8999])
def test_in_another_piece(gpu, dtype, code, n, t):
    check(gpu, dtype, code, [n], [9000], [t])
    check(gpu, dtype, code, [n], [9000], [t], bound=1 << 26)


@DTYPES
@CODES
@pytest.mark.parametrize("tree", [False, True], ids=["causal", "tree"])
@pytest.mark.parametrize("n", [12, 31, 60])
@pytest.mark.parametrize("bound", [None, 1 << 26], ids=["", "heads side by side"])
def test_new_keys_that_some_rows_see(gpu, dtype, code, tree, n, bound):
    check(gpu, dtype, code, [n, n, n], [0, 70, 500], [n // 2, 70 + n // 3, 500 + n // 2], tree=tree, bound=bound)
