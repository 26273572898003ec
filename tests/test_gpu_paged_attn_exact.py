"""Dense attention with huge logits that are exact in float: each row is the mean of the values of its largest ones, and its log-sum-exp is theirs."""
import math

import numpy as np
import pytest

import workloads as W
from cache_util import HALF, Cache, visible
from test_gpu_paged_attn_weights import BF, F32, LOOSE, call, gpu     # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("new,H,H_kv", [([1, 1], 8, 2), ([9, 9], 8, 2), ([40, 40], 8, 2), ([300, 300], 32, 8)])
@pytest.mark.parametrize("bound", [None, LOOSE], ids=["", "loose bound"])
@pytest.mark.parametrize("rounded", [False, True], ids=["", "rounded"])
@pytest.mark.parametrize("window,order", [(0, "any"), (0, "rising"), (0, "falling"), (90, "any"), (90, "negative")])
def test_logits_of_a_hundred_million(gpu, dtype, D, new, H, H_kv, bound, rounded, window, order):
    lens, n, G = [700, 650], new[0], H // H_kv
    c = Cache(dtype, H_kv, D, 16, lens, seed=n)
    rng = np.random.default_rng(D)
    m = [rng.integers(0, 256, (N, H_kv)) for N in lens]            # steps of 2^19: the next logit's weight is 0
    if order in ("rising", "falling"):
        m = [np.sort(x, axis=0)[::1 if order == "rising" else -1] for x in m]
    if order == "negative":
        m = [x - 300 for x in m]
    c.k_bits[:] = 0
    for b in range(2):
        k = np.zeros((lens[b], H_kv, D), np.float32)
        k[..., 5] = m[b] * 1024.0
        c.k_bits[c.slots(b)] = W.store(k, dtype)
    q = np.zeros((2 * n, H, D), np.float32)
    q[..., 5] = 4096.0
    out, lse, _, _ = call(gpu, c, H, new, rounded=rounded, window=window, bound=bound, sm=0.125, q=W.store(q, dtype))
    for b in range(2):
        for r in range(n):
            lo, hi = visible(lens[b], n, r, window)
            for kv in range(H_kv):
                z = m[b][lo:hi, kv] * (4096.0 * 1024.0 * 0.125)
                top = z == z.max()
                v = c.v[c.slots(b)[lo:hi][top], kv]
                want, size, count = v.mean(axis=0), np.abs(v).mean(axis=0), int(top.sum())
                rows = slice(kv * G, (kv + 1) * G)
                # weights are equal and exact but for their common factor: the sums' and the quotient's roundings, then the type's
                tol = size * (2 * count + 24) * 2.0 ** -24
                tol = tol + HALF[dtype] * (np.abs(want) + tol) + 1e-38
                assert np.all(np.abs(out[b * n + r, rows] - want) <= tol), (b, r, kv)
                assert np.all(np.abs(lse[b * n + r, rows] - (z.max() + math.log(count))) <= 4 * 2.0 ** -24 * (abs(z.max()) + 8)), (b, r, kv)
