"""Masks among the new tokens beside windows next to the largest int32: a window and a sequence's new tokens together pass it."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache, check_attention
from quant_util import QuantPages
from tree_util import attention, closure, random_tree, words_of

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32
LONGEST = 2 ** 31 - 1
DTYPES = pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
KINDS = pytest.mark.parametrize("code", [None, 0], ids=["pools", "int8"])


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


def check(ts, dtype, code, new, lens, window, H=8, H_kv=2, D=64):
    from paper_2411_02886_amd.runtime import to_host
    T, words, sm = sum(new), (max(new) + 31) // 32, 1 / math.sqrt(D)
    rng = np.random.default_rng(T)
    sees = [closure(random_tree(rng, n)) for n in new]
    q = W.store(rng.standard_normal((T, H, D), dtype=np.float32), dtype)
    mask, ind = dev(np.concatenate([words_of(s, words) for s in sees if len(s)]).view(np.int32)), dev(np.cumsum([0] + new).astype(np.int32))
    c = Cache(dtype, H_kv, D, 16, lens, seed=T) if code is None else QuantPages(dtype, code, H_kv, D, 16, lens, seed=T)
    held = c.problem(H, chunk=max(new), max_seq_len=LONGEST)
    p = held[0]
    out, lse = torch.full((T, H, D), 77, dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0"), torch.full((T, H), 55.0, device="cuda:0")
    n = (ts.ts_paged_attn_workspace_bytes if code is None else ts.ts_quant_attn_workspace_bytes)(p, T)
    ws = torch.full(((n + 255) // 256 * 64,), -1, dtype=torch.int32, device="cuda:0")
    if code is None:
        ts.ts_tree_attn(p, dev(q), ind, T, window, mask, sm, out, lse, ws)
    else:
        ts.ts_quant_attn(p, held[1], dev(q), ind, T, window, mask, sm, out, lse, ws)
    torch.cuda.synchronize()
    ref = attention(c, q, new, window, float(np.float32(sm)), sees, more=4 if code is not None else 0, tiny=0.0 if code is None else 2.0 ** -108)
    check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64), ref, (new, window))


@DTYPES
@KINDS
@pytest.mark.parametrize("new", [[3], [3, 5, 2], [90, 33, 7], [200]], ids=str)
def test_every_sequence_passes_it(gpu, dtype, code, new):
    check(gpu, dtype, code, new, [n + 300 for n in new], LONGEST - 1)


@DTYPES
@KINDS
@pytest.mark.parametrize("window", [LONGEST - 1, LONGEST - 4, LONGEST - 60, LONGEST - 90, LONGEST - 100])
def test_some_sequences_pass_it(gpu, dtype, code, window):
    check(gpu, dtype, code, [90, 1, 0, 5, 60, 3], [400, 33, 9, 5, 61, 1], window)      # (the last has fewer tokens than new ones)


def test_more_sequences_than_lanes(gpu):
    check(gpu, BF, 0, [2 + b % 9 for b in range(70)], [3 + b for b in range(70)], LONGEST - 6, H=6)      # (batch, heads and longest length: at most 2^40 together)
