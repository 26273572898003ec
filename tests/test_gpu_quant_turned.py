"""Codes and scales of turned keys bit for bit: those of the key that the type holds, which is the double's rounded to float and then to the type.  Left out are rows
with an element so near the middle of two floats that arithmetic in double may fall on either side; they have to be few."""
import numpy as np
import pytest

import workloads as W
from quant_util import QuantPages, encode

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


def turned(x, pos, inv_freq, adjacent, scale):
    """x [T][heads][D], pos [T]: (values, what arithmetic in double may be off).  The angle, a product that a double holds, is multiplied with 1 / 2 pi (rounded: 2^-54)
    and rounded, 2^-53: off by less than 2^-52 of it in all, here as in the reference at most 2^-51.  Sine, cosine, their products with the scale and with x and y,
    and the sum: eight roundings of 2^-53 and functions within two last bits, below 2^-49 of |scale| (|x| + |y|).  Angle 0 is exact: sine 0, cosine 1, and a double
    holds 1.25 x, which is the middle of two floats for many a float x."""
    out, tol, half = x.copy(), np.zeros_like(x), len(inv_freq)
    for i, f in enumerate(inv_freq.astype(np.float64)):
        a = pos * f
        e0, e1 = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        c, s = scale * np.cos(a)[:, None], scale * np.sin(a)[:, None]
        out[..., e0], out[..., e1] = x[..., e0] * c - x[..., e1] * s, x[..., e0] * s + x[..., e1] * c
        tol[..., e0] = tol[..., e1] = abs(scale) * (np.abs(x[..., e0]) + np.abs(x[..., e1])) * (2.0 ** -49 + 2.0 ** -51 * np.abs(a)[:, None]) * (a != 0)[:, None]
    return out, tol


def stored(w, tol, dtype):
    """(the rows as the type holds them, which rows are certain)."""
    low, high = (w - tol).astype(np.float32), (w + tol).astype(np.float32)
    return W.as_f32(W.store(w.astype(np.float32), dtype), dtype).astype(np.float64), (low == high).all(axis=-1)


@DTYPES
@CODES
@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("D,rotary", [(64, 64), (64, 24), (64, 26), (128, 128), (128, 32), (128, 2), (128, 120)])
@pytest.mark.parametrize("new", [[1, 2, 5], [70, 1, 90], [700]], ids=["few", "some", "many"])
def test_codes_of_turned_keys(gpu, dtype, code, adjacent, D, rotary, new):
    from paper_2411_02886_amd.runtime import to_device, to_host
    H, H_kv, T, scale = 6, 2, sum(new), 1.25
    rng = np.random.Generator(np.random.PCG64(rotary + T))
    lens = [n + 37 * b for b, n in enumerate(new)]
    c = QuantPages(dtype, code, H_kv, D, 16, lens, seed=T)
    p, quant = c.problem(H, chunk=max(new))
    rows = [W.store(rng.standard_normal((T, h, D), dtype=np.float32), dtype) for h in (H, H_kv, H_kv)]
    inv = (1e4 ** -(np.arange(rotary // 2) / (rotary // 2))).astype(np.float32)
    q_out = torch.zeros((T, H, D), dtype=torch.int16 if dtype == BF else torch.float32, device="cuda:0")
    gpu.ts_quant_append(p, quant, gpu.Rope(inv_freq=to_device(inv), adjacent=adjacent, scale=scale), *(to_device(x) for x in rows),
                        to_device(np.cumsum([0] + new).astype(np.int32)), T, None, q_out)
    torch.cuda.synchronize()
    codes, scales = c.read(quant)
    place = np.concatenate([np.arange(N - n, N) for n, N in zip(new, lens)])
    slot = np.concatenate([c.slots(b)[N - n:] for b, (n, N) in enumerate(zip(new, lens))])
    q, k, v = (W.as_f32(x, dtype).astype(np.float64) for x in rows)
    want, sure = stored(*turned(q, place, inv, adjacent, scale), dtype)
    got = W.as_f32(to_host(q_out, bits16=dtype == BF), dtype).astype(np.float64)
    assert np.array_equal(got[sure], want[sure]) and sure.mean() > 0.95
    want, sure = stored(*turned(k, place, inv, adjacent, scale), dtype)
    assert sure.mean() > 0.95, sure.mean()               # (angles up to 800: an element is uncertain with a chance of about 2^-16)
    for name, x, mine in (("k", want, sure), ("v", v, np.ones((T, H_kv), bool))):
        code_want, scale_want = encode(x, code)
        assert np.array_equal(scales[name][slot][mine], scale_want[mine]), name
        assert np.array_equal(codes[name][slot][mine], code_want[mine]), (name, int((codes[name][slot][mine] != code_want[mine]).sum()))
