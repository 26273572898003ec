"""ts_quant_append, ts_quant_read and ts_quant_pages_copy against the definition in 64 bits: codes and scales bit for bit where nothing is turned,
turned keys within a code's step, which slots are written, rows that hold zeros, tiny, huge and non-finite numbers, ties."""
import numpy as np
import pytest

import workloads as W
from cache_util import HALF
from quant_util import TOP, QuantPages, encode, step_of, to_code

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


def stored(x, dtype):
    bits = W.store(np.asarray(x, np.float32), dtype)
    if dtype == BF:
        bits[np.isnan(x)] = 0x7fc0
    return bits


def turned(x, pos, inv_freq, pair_axis, adjacent, scale):
    """x [T][heads][D] double, pos [axes][T]: the definition, and what arithmetic in double may be off: the angle by 2^-52 of it, a few roundings."""
    out, tol = x.copy(), np.zeros_like(x)
    half = len(inv_freq)
    for i in range(half):
        a = pos[pair_axis[i]].astype(np.float64) * float(inv_freq[i])
        e0, e1 = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        w = (x[..., e0] + 1j * x[..., e1]) * (scale * np.exp(1j * a))[:, None]
        out[..., e0], out[..., e1] = w.real, w.imag
        tol[..., e0] = tol[..., e1] = abs(scale) * (np.abs(x[..., e0]) + np.abs(x[..., e1])) * (2.0 ** -49 + 2.0 ** -51 * np.abs(a)[:, None])
    return out, tol


def case(ts, dtype, code, H, H_kv, D, P, new, lens, rotary=0, axes=0, adjacent=False, scale=1.0, packed=True, fused=True, in_place=False, far=0,
         seed=0, with_q=True, behind=0, max_seq_len=None, rows=None):
    from paper_2411_02886_amd.runtime import to_device, to_host
    rng = np.random.Generator(np.random.PCG64(seed))
    T = sum(new) + behind
    c = QuantPages(dtype, code, H_kv, D, P, lens, seed=seed + 1)
    p, quant = c.problem(H, chunk=max(1, max(new)), max_seq_len=max_seq_len)
    x = rng.standard_normal((T, (H + 2 * H_kv) * D), dtype=np.float32) if rows is None else rows
    qkv = stored(x, dtype)
    cut = [0, H * D, (H + H_kv) * D, (H + 2 * H_kv) * D]
    dev = to_device(qkv)
    q, k, v = (dev[:, a:b] for a, b in zip(cut, cut[1:]))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    half = rotary // 2
    inv = (1e4 ** -(np.arange(half) / max(1, half))).astype(np.float32)
    pair_axis = [int(rng.integers(0, max(1, axes))) for _ in range(half)]
    pos = rng.integers(-5 if far == 0 else far - 9, 3000 + far, size=(axes, T)).astype(np.int32) if axes else None
    rope = ts.Rope(inv_freq=to_device(inv), pair_axis=pair_axis, num_axes=max(1, axes), adjacent=adjacent, scale=scale) if rotary else None
    q_out = q if in_place else torch.full((T, H * D), 7, dtype=dev.dtype, device="cuda:0")
    ind = to_device(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None
    ts.ts_quant_append(p, quant, rope, q if with_q else None, k, v, ind, T, None if pos is None else to_device(pos), q_out if with_q else None)
    torch.cuda.synchronize()
    bits = dtype == BF
    place = np.concatenate([np.arange(N - n, N) for n, N in zip(new, lens)] + [np.zeros(behind, int)]).astype(np.int64)
    owner = np.concatenate([np.full(n, b) for b, n in enumerate(new)] + [np.full(behind, -1)]).astype(int)
    xs = W.as_f32(qkv, dtype).astype(np.float64)
    at, sc = pos if pos is not None else place[None], float(np.float32(scale))
    if with_q:
        got = W.as_f32(to_host(q_out, bits16=bits), dtype).astype(np.float64).reshape(T, H, D)
        want, tol = turned(xs[:, :cut[1]].reshape(T, H, D), at, inv, pair_axis, adjacent, sc)
        tol = tol + (HALF[dtype] + 2.0 ** -24 * bits) * (np.abs(want) + tol) + 2.0 ** -149
        mine = owner >= 0
        assert np.all(np.abs(got - want)[mine] <= tol[mine]), float(np.max((np.abs(got - want) / tol)[mine]))
        if behind and not in_place:
            assert np.all(to_host(q_out)[T - behind:] == 7)
    codes, scales = c.read(quant)
    limit = 1 << 30 if max_seq_len is None else max_seq_len
    written = np.zeros(codes["k"].shape[0], bool)
    k_want, k_tol = turned(xs[:, cut[1]:cut[2]].reshape(T, H_kv, D), at, inv, pair_axis, adjacent, sc)
    for r in range(T - behind):
        if not 0 <= place[r] < limit:
            continue
        s = c.slots(owner[r])[place[r]]
        written[s] = True
        want = encode(xs[r, cut[2]:].reshape(H_kv, D), code)
        assert np.array_equal(codes["v"][s], want[0]) and np.array_equal(scales["v"][s], want[1], equal_nan=True), r
        if rotary == 0:
            want = encode(xs[r, cut[1]:cut[2]].reshape(H_kv, D), code)
            assert np.array_equal(codes["k"][s], want[0]) and np.array_equal(scales["k"][s], want[1], equal_nan=True), r
            continue
        # a turned key: rounded to the type (and to float before), then to a code of a row whose largest value has been rounded as well
        w, tol = k_want[r], k_tol[r]
        tol = tol + (HALF[dtype] + 2.0 ** -24) * (np.abs(w) + tol)
        m = (np.abs(w) + tol).max(axis=-1, keepdims=True)
        tol = tol + 0.5 * step_of(np.abs(w) + tol, m, code) * (1 + 2.0 ** -20) + 2.0 ** -23 * np.abs(w)
        err = np.abs(c.values(codes["k"][s], scales["k"][s]) - w)
        assert np.all(err <= tol), (r, float(np.max(err / tol)))
    for n in "kv":
        assert np.array_equal(codes[n][~written], c.bytes[n][~written])
        assert np.array_equal(scales[n][~written], c.scales[n][~written], equal_nan=True)
    return written


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("rotary", [0, 2, 24, 26, 32, 64, 128])
def test_parts_of_a_head(gpu, dtype, code, D, adjacent, rotary):
    if rotary > D:
        pytest.skip("more than a head")
    case(gpu, dtype, code, 6, 2, D, 8, [3, 1, 9], [20, 1, 9], rotary, 2 if rotary else 0, adjacent=adjacent, seed=rotary)


@DTYPES
@CODES
@pytest.mark.parametrize("packed", [True, False], ids=["packed", "padded"])
@pytest.mark.parametrize("fused", [True, False], ids=["fused", "apart"])
@pytest.mark.parametrize("axes", [0, 1, 4])
def test_axes_and_rows(gpu, dtype, code, packed, fused, axes):
    new = [5, 0, 1, 12, 4] if packed else [4] * 5
    case(gpu, dtype, code, 8, 2, 64, 16, new, [40, 7, 1, 13, 16], 64, axes, packed=packed, fused=fused, seed=axes, scale=1.25, behind=2 if packed else 0)


@CODES
@pytest.mark.parametrize("H,H_kv,P", [(1, 1, 8), (28, 4, 16), (32, 32, 1), (1, 1, 1), (8, 8, 256), (128, 16, 16), (5, 1, 32)])
def test_head_layouts_and_pages(gpu, code, H, H_kv, P):
    for dtype in (BF, F32):
        case(gpu, dtype, code, H, H_kv, 128, P, [1, 2, 30], [700, 2, 31], 128, 1, seed=H)
        case(gpu, dtype, code, H, H_kv, 64, P, [1, 2, 30], [70, 2, 31], 0, 0, seed=H)


@DTYPES
@CODES
def test_far_positions(gpu, dtype, code):
    for far in (1 << 22, (1 << 31) - 4000):
        case(gpu, dtype, code, 4, 2, 64, 16, [7, 3], [50, 3], 64, 3, far=far, seed=4)


@DTYPES
@pytest.mark.parametrize("rotary,adjacent", [(64, False), (26, False), (64, True), (0, False)])
def test_in_place_and_without_queries(gpu, dtype, rotary, adjacent):
    axes = 1 if rotary else 0
    case(gpu, dtype, 0, 4, 2, 64, 16, [7, 3], [50, 3], rotary, axes, adjacent=adjacent, fused=False, in_place=True, seed=2)
    case(gpu, dtype, 1, 4, 2, 64, 16, [7, 3], [50, 3], rotary, axes, adjacent=adjacent, with_q=False, seed=2)


@DTYPES
@CODES
def test_places_that_do_not_exist_write_nothing(gpu, dtype, code):
    assert case(gpu, dtype, code, 4, 2, 64, 16, [5, 2, 3], [3, 0, 9], 64, 0, seed=3).sum() == 3 + 0 + 3
    assert case(gpu, dtype, code, 4, 2, 64, 16, [5, 2, 3], [30, 8, 9], 64, 0, seed=3, max_seq_len=8).sum() == 0 + 2 + 2


@DTYPES
@CODES
def test_rows_of_every_size_and_ties(gpu, dtype, code):
    """The code is that of the exact quotient: ties, which half a row's largest value and its odd multiples meet, go to the even one."""
    rng = np.random.Generator(np.random.PCG64(7))
    T, H, H_kv, D = 40, 2, 2, 64
    x = rng.standard_normal((T, (H + 2 * H_kv), D)).astype(np.float32)
    for r in range(T):
        x[r, 2:] *= np.float32(2.0) ** (-130 + 6 * r)                     # denormal numbers to 1e31
    x[3, 2:] = 0
    x[5, 2, 1:] = 0
    x[8, 3] = -0.0
    x[9, 2:] = 3e38 * np.sign(x[9, 2:])
    m = np.array([127.0, 254.0, 3.0, 1.0, 0.75, 448.0, 7.0, 1.9921875], np.float32)
    for i, top in enumerate(m):                                           # quotients that lie between two codes, exactly
        n = np.arange(D) - D // 2
        z = (2 * n + 1) / 2 if code == 0 else np.array([float(2 * (8 + j % 8) + 1) * 2.0 ** (j // 8 - 5) for j in range(D)]) * np.where(n % 2, 1, -1)
        row = (z * float(top) / TOP[code]).astype(np.float32)
        row = W.as_f32(W.store(row, dtype), dtype)
        row[0] = top
        x[20 + i, 2], x[20 + i, 3], x[20 + i, 4], x[20 + i, 5] = row, -row, row * 0.5, row * 1024
        x[20 + i, 4, 5] = x[20 + i, 4, 0] / 2                             # 63.5 of 127
    case(gpu, dtype, code, H, H_kv, D, 16, [T], [T + 3], rows=x.reshape(T, -1), fused=False)


def test_the_reference_codes_are_those_of_the_format():
    z = torch.tensor([0.0, 1.0, 17.0, 18.0, 19.0, 0.001953125, 0.0009765625, 0.003, -25.0, -27.0, 240.0, 247.9, 248.0, 447.0, 448.0, -0.0])
    assert np.array_equal(to_code(z.double().numpy(), 1), z.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


@DTYPES
@CODES
@pytest.mark.parametrize("rotary", [0, 64])
def test_rows_that_are_not_finite_read_back_as_nan_and_no_other_row_does(gpu, dtype, code, rotary):
    from paper_2411_02886_amd.runtime import to_device, to_host
    rng = np.random.Generator(np.random.PCG64(1))
    T, H_kv, D = 6, 4, 64
    c = QuantPages(dtype, code, H_kv, D, 16, [9], seed=3)
    p, quant = c.problem(8, chunk=T)
    k, v = (rng.standard_normal((T, H_kv, D)).astype(np.float32) for _ in "kv")
    k[1, 2, 5], k[2, 0, 63], v[3, 1, 0], v[4, 3, 40] = np.nan, np.inf, -np.inf, np.nan
    dev = [to_device(stored(x, dtype)) for x in (k, v)]
    rope = gpu.Rope(inv_freq=to_device(np.full(rotary // 2, 0.5, np.float32))) if rotary else None
    gpu.ts_quant_append(p, quant, rope, None, dev[0], dev[1], None, T, None, None)
    out = [torch.zeros_like(x) for x in dev]
    gpu.ts_quant_read(p, quant, None, T, out[0], out[1])
    torch.cuda.synchronize()
    for got, x in zip(out, (k, v)):
        got = W.as_f32(to_host(got, bits16=dtype == BF), dtype)
        bad = ~np.isfinite(x).all(axis=-1)
        assert bad.sum() == 2 and np.isnan(got[bad]).all() and np.isfinite(got[~bad]).all()
    codes, scales = c.read(quant)
    assert not codes["k"][c.slots(0)[3:]][~np.isfinite(k).all(axis=-1)].any() and np.isnan(scales["v"][c.slots(0)[3:]]).sum() == 2


def read(ts, dtype, code, H_kv, D, P, new, lens, packed=True, seed=0, max_seq_len=None, behind=0, what="kv"):
    from paper_2411_02886_amd.runtime import to_device, to_host
    c = QuantPages(dtype, code, H_kv, D, P, lens, seed=seed)
    p, quant = c.problem(H_kv, chunk=max(1, max(new)), max_seq_len=max_seq_len)
    T = sum(new) + behind
    es = torch.int16 if dtype == BF else torch.float32
    out = {n: torch.full((T, H_kv, D), 7, dtype=es, device="cuda:0") if n in what else None for n in "kv"}
    ts.ts_quant_read(p, quant, to_device(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None, T, out["k"], out["v"])
    torch.cuda.synchronize()
    limit = 1 << 30 if max_seq_len is None else max_seq_len
    for n in what:
        got, row = to_host(out[n], bits16=dtype == BF), 0
        for b, m in enumerate(new):
            for i in range(m):
                t = int(lens[b]) - m + i
                want = np.zeros((H_kv, D), np.float32)
                if 0 <= t < limit:
                    s = c.slots(b)[t]
                    codes, scales = c.bytes[n][s], c.scales[n][s]
                    want = c.values(codes, np.ones_like(scales)).astype(np.float32) * scales[:, None]
                assert np.array_equal(got[row], W.store(want, dtype)), (n, b, i)
                row += 1
        assert np.all(got[row:] == 7)


@DTYPES
@CODES
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H_kv,P", [(1, 1), (1, 8), (2, 16), (8, 16), (32, 4), (16, 64)])
def test_read(gpu, dtype, code, D, H_kv, P):
    read(gpu, dtype, code, H_kv, D, P, [3, 0, 17, 1, 40], [20, 5, 17, 1, 133], seed=P, behind=2)
    read(gpu, dtype, code, H_kv, D, P, [5, 5, 5], [3, 5, 70], packed=False, seed=P)            # the first rows stand for no token: 0


@DTYPES
def test_read_of_whole_sequences_one_pool_and_bounds(gpu, dtype):
    read(gpu, dtype, 0, 2, 64, 16, [1000, 0, 333], [1000, 0, 333], what="k")
    read(gpu, dtype, 1, 2, 64, 16, [1000, 1, 333], [1000, 1, 333], what="v", max_seq_len=900)


def test_nothing_to_do(gpu):
    c = QuantPages(BF, 0, 2, 64, 16, [5], seed=1)
    p, quant = c.problem(8)
    gpu.ts_quant_append(p, quant, None, None, None, None, None, 0, None, None)
    gpu.ts_quant_read(p, quant, None, 0, None, None)
    z = torch.zeros(1, dtype=torch.int32, device="cuda:0")
    gpu.ts_quant_pages_copy(p, quant, z, z, 0, 1)
    torch.cuda.synchronize()


def test_many_sequences_and_a_long_prompt(gpu):
    rng = np.random.Generator(np.random.PCG64(3))
    lens = rng.integers(0, 9, size=1500).tolist()
    new = [int(rng.integers(0, n + 1)) for n in lens]
    case(gpu, BF, 0, 2, 1, 64, 8, new, lens, 64, 1, seed=9)
    case(gpu, F32, 1, 4, 2, 64, 16, [2500], [3001], 64, 3, seed=10)
    read(gpu, BF, 1, 1, 64, 8, new, lens, seed=9)


@pytest.mark.parametrize("P,H_kv,D", [(16, 8, 128), (1, 1, 64), (1, 2, 64), (8, 1, 64), (64, 2, 128)])
def test_pages_copy(gpu, P, H_kv, D):
    from paper_2411_02886_amd.runtime import to_device
    c = QuantPages(BF, 1, H_kv, D, P, [9 * P], seed=5, spare=6)
    p, quant = c.problem(H_kv)
    n = c.num_pages
    src = [int(c.pages[0]), int(c.pages[1]), int(c.pages[1]), -1, 3, n, int(c.pages[4]), int(c.pages[2])]
    dst = [int(c.spare[0]), int(c.spare[1]), int(c.spare[2]), 0, -1, 1, n + 5, int(c.pages[2])]
    gpu.ts_quant_pages_copy(p, quant, to_device(np.array(src, np.int32)), to_device(np.array(dst, np.int32)), len(src), n)
    torch.cuda.synchronize()
    codes, scales = c.read(quant)
    for name in "kv":
        a, b = c.bytes[name].reshape(n, -1).copy(), c.scales[name].reshape(n, -1).copy()
        for i in range(3):
            a[dst[i]], b[dst[i]] = a[src[i]], b[src[i]]
        assert np.array_equal(codes[name].reshape(n, -1), a) and np.array_equal(scales[name].reshape(n, -1), b, equal_nan=True)


@CODES
def test_captured_calls_read_lengths_and_positions_when_they_run(gpu, code):
    from paper_2411_02886_amd.runtime import to_device
    c = QuantPages(BF, code, 2, 64, 16, [40, 17], seed=1)
    p, quant = c.problem(4)
    rng = np.random.default_rng(0)
    q, k, v = (to_device(W.store(rng.standard_normal((2, h, 64), dtype=np.float32), BF)) for h in (4, 2, 2))
    rope = gpu.Rope(inv_freq=to_device((1e4 ** -(np.arange(32) / 32)).astype(np.float32)))
    pos, lens = to_device(np.array([[9, 12]], np.int32)), p._keep[4]
    held = [t.clone() for t in quant._keep]
    out = [torch.zeros_like(t) for t in (q, k, v)]

    def call():
        gpu.ts_quant_append(p, quant, rope, q, k, v, None, 2, pos, out[0])
        gpu.ts_quant_read(p, quant, None, 2, out[1], out[2])

    def reset():
        for t, h in zip(quant._keep, held):
            t.copy_(h)
        for t in out:
            t.zero_()

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call()
    for rep in range(4):
        reset()
        torch.cuda.synchronize()
        g.replay(); torch.cuda.synchronize()
        got = [t.clone() for t in (*out, *quant._keep)]
        reset()
        call(); torch.cuda.synchronize()
        for a, b in zip(got, (*out, *quant._keep)):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), rep
        pos += 3
        lens -= 1
