"""References in 64 bits of the calls that fill, attend and move a paged cache, and error bounds that follow from the arithmetic."""
import numpy as np

import workloads as W

HALF = {W.BF16: 2.0 ** -8, W.F32: 2.0 ** -24}       # half a step of the storage type, relative


class Cache:
    """Random pools and a page table for sequences of the given lengths; `spare` pages that no sequence owns.  Every slot that
    holds no token of a sequence is NaN: no call may let it into a result."""

    def __init__(self, dtype, H_kv, D, P, lens, seed, spare=2, scale=1.0):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.dtype, self.H_kv, self.D, self.P, self.B = dtype, H_kv, D, P, len(lens)
        self.lens = np.asarray(lens, dtype=np.int32)
        need = [max(0, -(-int(n) // P)) for n in lens]
        self.indptr = np.cumsum([0] + need).astype(np.int32)
        perm = rng.permutation(sum(need) + spare).astype(np.int32)
        self.pages, self.spare = perm[:sum(need)], perm[sum(need):]
        shape = ((sum(need) + spare) * P, H_kv, D)
        nan = np.full(shape, np.nan, dtype=np.float32)
        self.k, self.v = nan.copy(), nan.copy()
        for b in range(self.B):
            at = self.slots(b)
            self.k[at] = scale * rng.standard_normal((len(at), H_kv, D), dtype=np.float32)
            self.v[at] = rng.standard_normal((len(at), H_kv, D), dtype=np.float32)
        self.k_bits, self.v_bits = W.store(self.k, dtype), W.store(self.v, dtype)
        if dtype == W.BF16:                             # NaN as bits: rounding by integers would make something else of it
            for bits, x in ((self.k_bits, self.k), (self.v_bits, self.v)):
                bits[np.isnan(x)] = 0x7fc0
        self.k, self.v = W.as_f32(self.k_bits, dtype).astype(np.float64), W.as_f32(self.v_bits, dtype).astype(np.float64)

    def slots(self, b, n=None):
        t = np.arange(int(self.lens[b]) if n is None else n)
        return self.pages[self.indptr[b] + t // self.P].astype(np.int64) * self.P + t % self.P

    def problem(self, H, chunk=1, max_seq_len=None, **kw):
        """(Problem, k_pool, v_pool) on the GPU."""
        import paper_2411_02886_amd as ts
        from paper_2411_02886_amd.runtime import to_device
        pool = (-1, self.P, self.H_kv, self.D)
        k, v = to_device(self.k_bits.reshape(pool)), to_device(self.v_bits.reshape(pool))
        pages = self.pages if self.pages.size else np.zeros(1, np.int32)
        p = ts.Problem(batch=self.B, chunk=chunk, num_q_heads=H, num_kv_heads=self.H_kv, head_dim=self.D, page_size=self.P,
                       max_seq_len=max(1, int(self.lens.max())) if max_seq_len is None else max_seq_len, dtype=self.dtype,
                       k_pool=k, v_pool=v, page_indptr=to_device(self.indptr), page_indices=to_device(pages),
                       seq_lens=to_device(self.lens), **kw)
        return p, k, v


def visible(N, n, c, window):
    """First and one past the last token that new token c of n sees in a sequence of N."""
    x = N - n + c
    return (max(0, x - window + 1) if window else 0), x + 1


def attention(cache, q, new, window, sm, weights_rounded):
    """q [T][H][D] stored; new: new tokens per sequence.  (out, lse, bound on out, bound on lse), rows in order.

    The bounds.  A logit is a sum of D products, each rounded at most once on its way (bf16 products are exact in float): off by at most
    (D + 1) 2^-24 sum |q k| sm, plus 4 roundings of its own size (scale, base 2, reference): call it e.  A weight is off by a factor e^(2 e)
    and 4 roundings, the sums of N weights or weighted values by N + 8 roundings more (splits joined: 8 more).  So with A = sum p |v|:
    out is off by A (2 e + (2 N + 32) 2^-24), and A 2^-8 where a weight is rounded to bf16, then by half a step of its type; lse by
    e + (N + 16) 2^-24 and four roundings of its size."""
    q32 = W.as_f32(q, cache.dtype).astype(np.float64)
    T, H, D = q32.shape
    G, u = H // cache.H_kv, 2.0 ** -24
    out, lse = np.zeros((T, H, D)), np.full((T, H), -np.inf)
    tol_o, tol_l = np.zeros((T, H, D)), np.zeros((T, H))
    row = 0
    for b, n in enumerate(new):
        N = int(cache.lens[b])
        at = cache.slots(b)
        for kv in range(cache.H_kv):
            k, v = cache.k[at, kv], cache.v[at, kv]
            hs = slice(kv * G, (kv + 1) * G)
            for c in range(n):
                lo, hi = visible(N, n, c, window)
                if hi <= lo:
                    continue
                kk, vv, qq = k[lo:hi], v[lo:hi], q32[row + c, hs]
                z = (qq @ kk.T) * sm
                e = (np.abs(qq) @ np.abs(kk).T).max(axis=1) * abs(sm) * (D + 1) * u + 6 * u * np.abs(z).max(axis=1) + 8 * u
                m = z.max(axis=1, keepdims=True)
                p = np.exp(z - m)
                l = p.sum(axis=1, keepdims=True)
                out[row + c, hs] = p @ vv / l
                A = p @ np.abs(vv) / l
                lse[row + c, hs] = (m + np.log(l))[:, 0]
                M = hi - lo
                rel = np.expm1(2 * e) + (2 * M + 32) * u + (2.0 ** -8 if weights_rounded[b] else 0.0)
                tol_o[row + c, hs] = A * rel[:, None] + HALF[cache.dtype] * (np.abs(out[row + c, hs]) + A * rel[:, None]) + 1e-38
                tol_l[row + c, hs] = e + (M + 16) * u + 4 * u * np.abs(lse[row + c, hs])
        row += n
    return out, lse, tol_o, tol_l


def check_attention(got_out, got_lse, ref, label):
    out, lse, tol_o, tol_l = ref
    empty = np.isinf(lse)
    assert np.array_equal(np.isneginf(got_lse), empty), label
    assert not np.any(got_out[empty]), label
    err = np.abs(got_out - out)
    assert np.all(err <= tol_o), (label, "out", float((err / tol_o).max()), np.unravel_index(np.argmax(err / tol_o), err.shape))
    err = np.abs(np.where(empty, 0, got_lse) - np.where(empty, 0, lse))
    assert np.all(err <= np.maximum(tol_l, 1e-30)), (label, "lse", float((err / np.maximum(tol_l, 1e-30)).max()))
