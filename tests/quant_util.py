"""References in 64 bits of the 8-bit cache: codes, scales, and pages filled with them."""
import numpy as np

import workloads as W

TOP = {0: 127.0, 1: 448.0}                                   # TS_INT8, TS_E4M3
# the 127 values of e4m3 from 0 up: four bits of exponent, three behind the point, no infinities (code 127 is NaN)
E4M3 = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (8 + (c & 7)) * 2.0 ** ((c >> 3) - 10) for c in range(127)])


def to_code(z, code):
    """Codes (bytes) of quotients: nearest, ties to the even one."""
    if code == 0:
        return np.rint(z).astype(np.int8).view(np.uint8)
    a = np.abs(z)
    up = np.clip(np.searchsorted(E4M3, a), 0, 126)           # first value >= a
    down = np.maximum(up - 1, 0)
    lo, hi = a - E4M3[down], E4M3[up] - a                    # (exact: neighbours within a factor of two, or small multiples of a step)
    c = np.where((hi < lo) | ((hi == lo) & (up % 2 == 0)), up, down)
    return (c | np.where(np.signbit(z), 128, 0)).astype(np.uint8)


def of_code(c, code):
    if code == 0:
        return c.view(np.int8).astype(np.float64)
    v = np.where((c & 127) == 127, np.nan, E4M3[np.minimum(c & 127, 126)])
    return np.where(c & 128, -v, v)


def encode(rows, code):
    """(codes, scales) of rows [..., D] of stored values, by the definition."""
    x = np.asarray(rows, dtype=np.float64)
    m = np.abs(x).max(axis=-1, keepdims=True)
    bad = ~np.isfinite(x).all(axis=-1, keepdims=True)
    with np.errstate(all="ignore"):
        z = np.where((m > 0) & ~bad, x * TOP[code] / m, 0.0)
    return to_code(z, code), np.where(bad, np.nan, m / TOP[code])[..., 0].astype(np.float32)


def step_of(value, m, code):
    """The largest step between codes around a value of a row whose largest is m."""
    if code == 0:
        return np.broadcast_to(m / 127, value.shape)
    z = np.maximum(np.abs(value) / np.maximum(m / 448, 1e-300), 2.0 ** -6)
    return 2.0 ** (np.floor(np.log2(z)) + 1 - 3) * m / 448    # one binade up, should it lie at its end


class QuantPages:
    """Random 8-bit pages and a page table for sequences of the given lengths.  Slots that hold no token of a sequence have scale NaN and codes
    255: no call may let them into a result."""

    def __init__(self, dtype, code, H_kv, D, P, lens, seed, spare=2, scale=1.0, fill=True):
        rng = np.random.Generator(np.random.PCG64(seed))
        self.dtype, self.code, self.H_kv, self.D, self.P, self.B = dtype, code, H_kv, D, P, len(lens)
        self.lens = np.asarray(lens, dtype=np.int32)
        need = [max(0, -(-int(n) // P)) for n in lens]
        self.indptr = np.cumsum([0] + need).astype(np.int32)
        perm = rng.permutation(sum(need) + spare).astype(np.int32)
        self.pages, self.spare, self.num_pages = perm[:sum(need)], perm[sum(need):], sum(need) + spare
        self.bytes = {n: np.full((self.num_pages * P, H_kv, D), 255, np.uint8) for n in "kv"}
        self.scales = {n: np.full((self.num_pages * P, H_kv), np.nan, np.float32) for n in "kv"}
        for b in range(self.B if fill else 0):
            at = self.slots(b)
            for n, size in (("k", scale), ("v", 1.0)):
                x = W.as_f32(W.store(size * rng.standard_normal((len(at), H_kv, D), dtype=np.float32), dtype), dtype)
                self.bytes[n][at], self.scales[n][at] = encode(x, code)
        self.k, self.v = (self.values(self.bytes[n], self.scales[n]) for n in "kv")

    def values(self, codes, scales):
        return of_code(codes, self.code) * scales[..., None].astype(np.float64)

    def slots(self, b, n=None):
        t = np.arange(int(self.lens[b]) if n is None else n)
        return self.pages[self.indptr[b] + t // self.P].astype(np.int64) * self.P + t % self.P

    def problem(self, H, chunk=1, max_seq_len=None, **kw):
        """(Problem, QuantCache) on the GPU."""
        import torch

        import paper_2411_02886_amd as ts
        from paper_2411_02886_amd.runtime import to_device
        codes = [torch.from_numpy(self.bytes[n].reshape(-1, self.P, self.H_kv, self.D)).to("cuda:0") for n in "kv"]
        scale = [to_device(self.scales[n].reshape(-1, self.P, self.H_kv).transpose(0, 2, 1)) for n in "kv"]
        c = ts.QuantCache(k_codes=codes[0], v_codes=codes[1], k_scale=scale[0], v_scale=scale[1], format=self.code)
        pages = self.pages if self.pages.size else np.zeros(1, np.int32)
        p = ts.Problem(batch=self.B, chunk=chunk, num_q_heads=H, num_kv_heads=self.H_kv, head_dim=self.D, page_size=self.P,
                       max_seq_len=max(1, int(self.lens.max())) if max_seq_len is None else max_seq_len, dtype=self.dtype,
                       k_pool=None, v_pool=None, page_indptr=to_device(self.indptr), page_indices=to_device(pages),
                       seq_lens=to_device(self.lens), **kw)
        return p, c

    def read(self, c):
        """(codes, scales) by slot of a QuantCache on the GPU, for "k" and "v"."""
        from paper_2411_02886_amd.runtime import to_host
        kc, vc, ks, vs = (to_host(t) for t in c._keep)
        flat = lambda s: np.ascontiguousarray(s.transpose(0, 2, 1)).reshape(-1, self.H_kv)
        return {"k": kc.reshape(-1, self.H_kv, self.D), "v": vc.reshape(-1, self.H_kv, self.D)}, {"k": flat(ks), "v": flat(vs)}
