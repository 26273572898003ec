"""Dense attention where a visible key is no number: the rows that see it come out NaN, with NaN for the log-sum-exp, not as rows that see nothing."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import Cache, attention, check_attention
from test_gpu_paged_attn_weights import BF, F32, LOOSE, call, gpu     # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

# new tokens and heads: a single token; tiles of 32 rows; large tiles, by a workgroup each and in shares
SHAPES = [([1, 1], 8, 2), ([9, 9], 8, 2), ([40, 40], 8, 2), ([300, 300], 32, 8)]


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,H,H_kv", SHAPES)
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
@pytest.mark.parametrize("rounded", [False, True], ids=["", "rounded"])
def test_rows_that_see_a_key_that_is_no_number(gpu, dtype, D, new, H, H_kv, bound, rounded):
    lens, n = [700, 650], new[0]
    c = Cache(dtype, H_kv, D, 16, lens, seed=n)
    ref_k = c.k.copy()
    # sequence 0: a cached key of one KV head; sequence 1: the key of its new token in the middle, which the tokens before do not see
    nan = 0x7fc0 if dtype == BF else np.nan
    c.k_bits[c.slots(0)[100], 1] = nan
    c.k_bits[c.slots(1)[650 - n + n // 2], 0] = nan
    out, lse, q, sm = call(gpu, c, H, new, rounded=rounded, bound=bound)
    G = H // H_kv
    want = np.zeros((2 * n, H), bool)
    want[:n, G:2 * G] = True
    want[n + n // 2:, :G] = True
    assert np.array_equal(np.isnan(lse), want)
    assert np.array_equal(np.isnan(out), np.broadcast_to(want[..., None], out.shape))
    c.k = ref_k
    ref = attention(c, q, new, 0, sm, [rounded and dtype == BF and n * G > 32] * 2)
    out[want], lse[want] = ref[0][want], ref[1][want]
    check_attention(out, lse, ref, n)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new,H,H_kv", SHAPES)
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
def test_infinite_logits(gpu, dtype, new, H, H_kv, bound):
    """Above all others: inf - inf, no number.  Below all others: weight 0, as that of a logit of -1e30."""
    D, n = 64, new[0]
    q = W.store(np.abs(np.random.default_rng(1).standard_normal((2 * n, H, D))).astype(np.float32), dtype)
    for value in (np.inf, -np.inf):
        c = Cache(dtype, H_kv, D, 16, [700, 650], seed=n)
        at = [c.slots(0)[100], c.slots(1)[0]]
        c.k_bits[at] = {np.inf: 0x7f80, -np.inf: 0xff80}[value] if dtype == BF else value
        out, lse, _, _ = call(gpu, c, H, new, bound=bound, q=q)
        if value > 0:
            assert np.isnan(out).all() and np.isnan(lse).all()
        else:
            c.k_bits[at] = W.store(np.full((2, H_kv, D), -1e30, np.float32), dtype)
            same = call(gpu, c, H, new, bound=bound, q=q)
            assert np.isfinite(out).all() and np.array_equal(out, same[0]) and np.array_equal(lse, same[1])
