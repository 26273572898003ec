"""References in 64 bits of attention with a mask among the new tokens, over plain and 8-bit caches, and random trees."""
import numpy as np

import workloads as W
from cache_util import HALF


def random_tree(rng, n, near=9, roots=False):
    """Parents: each node follows one of the `near` before it; roots: several nodes may begin a path."""
    return np.array([int(rng.integers(max(-1 if roots or i == 0 else 0, i - near), i)) if i else -1 for i in range(n)], dtype=np.int32)


def closure(parents):
    """sees[i][j]: j is i or leads to it.  What cannot be a parent makes a root."""
    n = len(parents)
    sees = np.eye(n, dtype=bool)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            sees[i] |= sees[p]
    return sees


def words_of(sees, words):
    """[n][words] uint32 of bool [n][n]; bits beyond the words are dropped."""
    n = len(sees)
    bits = np.zeros((n, max(words * 32, n)), dtype=np.uint64)
    bits[:, :n] = sees
    return (bits[:, :words * 32].reshape(n, words, 32) << np.arange(32, dtype=np.uint64)).sum(axis=-1).astype(np.uint32)


def attention(cache, q, new, window, sm, sees=None, more=0, tiny=0.0):
    """q [T][H][D] stored; sees: per sequence bool [n][n], or None: causal.  (out, lse, bound on out, bound on lse), rows in order; `cache` holds k, v in 64
    bits.  Bounds as in cache_util.attention, with `more` roundings of a logit and of a weight (scales), and `tiny` of output for each key that a row sees: what is
    lost where weights leave the range of float.  bf16: a weight may be multiplied as two bf16 numbers, each rounded to nearest.  With 2^e <= w < 2^(e+1) the first's
    half step is 2^(e-8); what it leaves is that (a bf16 number) or has an exponent of e - 9 at most, and the second's half step is 2^(e-17) <= 2^-17 w."""
    q64 = W.as_f32(q, cache.dtype).astype(np.float64)
    T, H, D = q64.shape
    G, u, row = H // cache.H_kv, 2.0 ** -24, 0
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    tol_o, tol_l = np.zeros((T, H, D)), np.zeros((T, H))
    for b, n in enumerate(new):
        N = int(cache.lens[b])
        base, at = N - n, cache.slots(b)
        t, c = np.arange(N), np.arange(n)
        if sees is None:
            seen = t[None, :] <= base + c[:, None]
            if window:
                seen &= t[None, :] > base + c[:, None] - window
        else:
            seen = np.broadcast_to(t[None, :] < base, (n, N)).copy()
            if window:
                seen &= t[None, :] >= base + sees[b].sum(axis=1)[:, None] - window
            first = max(base, 0)
            seen[:, first:] = sees[b][:, first - base:]
        for kv in range(cache.H_kv if n and N else 0):
            k, v = cache.k[at, kv], cache.v[at, kv]
            used = seen.any(axis=0)                          # (what nobody sees may be anything)
            k, v = np.where(used[:, None], k, 0.0), np.where(used[:, None], v, 0.0)
            lost = (seen & np.isnan(v).any(axis=1)).any(axis=1)          # rows that see a value which is no number; it is nothing to the others
            v = np.where(np.isnan(v).any(axis=1, keepdims=True), 0.0, v)
            for g in range(G):
                h = kv * G + g
                qq = q64[row:row + n, h]
                z = (qq @ k.T) * sm
                az = np.where(seen, np.abs(qq) @ np.abs(k).T, 0.0)
                e = az.max(axis=1) * abs(sm) * (D + 1) * u + (6 + more) * u * np.where(seen, np.abs(z), 0.0).max(axis=1) + 8 * u
                z = np.where(seen, z, -np.inf)
                m = z.max(axis=1, keepdims=True)
                some = np.isfinite(m[:, 0])
                p = np.exp(z - np.where(np.isfinite(m), m, 0.0))
                l = p.sum(axis=1, keepdims=True)
                d = np.where(l > 0, l, 1.0)
                o, A, M = p @ v / d, p @ np.abs(v) / d, seen.sum(axis=1)
                rel = (np.expm1(2 * e) + (2 * M + 32 + more) * u + (2.0 ** -17 if cache.dtype == W.BF16 else 0.0))[:, None]
                out[row:row + n, h] = np.where(lost[:, None], np.nan, o)
                with np.errstate(divide="ignore"):
                    lse[row:row + n, h] = np.where(some, np.where(some, m[:, 0], 0.0) + np.log(l[:, 0]), -np.inf)
                tol_o[row:row + n, h] = A * rel + HALF[cache.dtype] * (np.abs(o) + A * rel) + 1e-38 + tiny * M[:, None]
                tol_l[row:row + n, h] = e + (M + 16) * u + 4 * u * np.abs(np.where(some, lse[row:row + n, h], 0.0))
        row += n
    return out, lse, tol_o, tol_l
