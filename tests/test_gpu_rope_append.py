"""ts_rope_append against complex multiplication in 64 bits: axes, pairings, parts of a head, strides, in place, far positions, and
which places of the pool are written."""
import numpy as np
import pytest

import workloads as W
from cache_util import HALF, Cache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

BF, F32 = W.BF16, W.F32


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def turned(x, pos, inv_freq, pair_axis, adjacent, scale):
    """x [T][heads][D] double, pos [axes][T]: the definition, and a bound on what float arithmetic may be off: the angle's
    own rounding (2^-53 of it, twice), cosine and sine by 2^-22 (argument rounded to float, function, factor), two products and a sum."""
    out, tol = x.copy(), np.zeros_like(x)
    half = len(inv_freq)
    for i in range(half):
        a = pos[pair_axis[i]].astype(np.float64) * float(inv_freq[i])
        e0, e1 = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        w = (x[..., e0] + 1j * x[..., e1]) * (scale * np.exp(1j * a))[:, None]
        out[..., e0], out[..., e1] = w.real, w.imag
        size = abs(scale) * (np.abs(x[..., e0]) + np.abs(x[..., e1]))
        tol[..., e0] = tol[..., e1] = size * (2.0 ** -22 + 2.0 ** -52 * np.abs(a)[:, None] + 3 * 2.0 ** -24)
    return out, tol


def case(ts, dtype, H, H_kv, D, P, new, lens, rotary, axes, adjacent=False, scale=1.0, packed=True, fused=True, in_place=False,
         far=0, seed=0, what="qkv", freqs=None, behind=0, max_seq_len=None):
    from paper_2411_02886_amd.runtime import to_device, to_host
    rng = np.random.Generator(np.random.PCG64(seed))
    T = sum(new) + behind
    c = Cache(dtype, H_kv, D, P, lens, seed=seed + 1)
    p, kp, vp = c.problem(H, chunk=max(1, max(new)), max_seq_len=max_seq_len)
    qkv = W.store(rng.standard_normal((T, (H + 2 * H_kv) * D), dtype=np.float32), dtype)
    cut = [0, H * D, (H + H_kv) * D, (H + 2 * H_kv) * D]
    dev = to_device(qkv)
    q, k, v = (dev[:, a:b] for a, b in zip(cut, cut[1:]))
    if not fused:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    half = rotary // 2
    inv = (1e4 ** -(np.arange(half) / max(1, half))).astype(np.float32) if freqs is None else freqs
    pair_axis = [int(rng.integers(0, max(1, axes))) for _ in range(half)]
    pos = rng.integers(-5 if far == 0 else far - 9, 3000 + far, size=(axes, T)).astype(np.int32) if axes else None
    rope = ts.Rope(inv_freq=to_device(inv), pair_axis=pair_axis, num_axes=max(1, axes), adjacent=adjacent, scale=scale) if rotary else None
    q_out = q if in_place else torch.full((T, H * D), 7, dtype=dev.dtype, device="cuda:0")
    ind = to_device(np.cumsum([0] + list(new)).astype(np.int32)) if packed else None
    use_q, use_k = "q" in what, "k" in what
    ts.ts_rope_append(p, rope, q if use_q else None, k if use_k else None, v if use_k else None, ind, T,
                      None if pos is None else to_device(pos), q_out if use_q else None)
    torch.cuda.synchronize()
    bits = dtype == BF
    # places
    place = np.concatenate([np.arange(N - n, N) for n, N in zip(new, lens)] + [np.zeros(behind, int)]).astype(np.int64)
    owner = np.concatenate([np.full(n, b) for b, n in enumerate(new)] + [np.full(behind, -1)]).astype(int)
    x = W.as_f32(qkv, dtype).astype(np.float64)
    at = pos if pos is not None else place[None]
    sc = float(np.float32(scale))
    # a negative place turns by itself too (nothing else is given); rows of no sequence are not turned
    got = W.as_f32(to_host(q_out, bits16=bits), dtype).astype(np.float64).reshape(T, H, D)
    want, tol = turned(x[:, :cut[1]].reshape(T, H, D), at, inv, pair_axis, adjacent, sc)
    tol = tol + HALF[dtype] * (np.abs(want) + tol)
    mine = owner >= 0
    if use_q:
        assert np.all(np.abs(got - want)[mine] <= tol[mine]), float(np.max((np.abs(got - want) / np.maximum(tol, 1e-300))[mine]))
        if rotary < D:
            assert np.array_equal(got[mine][..., rotary:], x[:, :cut[1]].reshape(T, H, D)[mine][..., rotary:])
        if behind and not in_place:
            assert np.all(to_host(q_out)[T - behind:] == 7)
    kg, vg = (to_host(t, bits16=bits).reshape(-1, H_kv, D) for t in (kp, vp))
    written = np.zeros(kg.shape[0], bool)
    if use_k:
        want, tol = turned(x[:, cut[1]:cut[2]].reshape(T, H_kv, D), at, inv, pair_axis, adjacent, sc)
        tol = tol + HALF[dtype] * (np.abs(want) + tol)
        vb = qkv[:, cut[2]:].reshape(T, H_kv, D)
        for r in range(T - behind):
            if place[r] < 0:
                continue
            s = c.slots(owner[r])[place[r]]
            written[s] = True
            err = np.abs(W.as_f32(kg[s], dtype).astype(np.float64) - want[r])
            assert np.all(err <= tol[r]), (r, float(np.max(err / np.maximum(tol[r], 1e-300))))
            assert np.array_equal(vg[s], vb[r]), r
    # nothing else of the pools has changed, NaN included
    view = np.uint16 if bits else np.uint32
    for now, was in ((kg, c.k_bits), (vg, c.v_bits)):
        assert np.array_equal(np.ascontiguousarray(now[~written]).view(view), np.ascontiguousarray(was[~written]).view(view))
    return written


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("rotary", [2, 24, 26, 32, 62, 64, 128])
def test_parts_of_a_head(gpu, dtype, D, adjacent, rotary):
    if rotary > D:
        pytest.skip("more than a head")
    case(gpu, dtype, 6, 2, D, 8, [3, 1, 9], [20, 1, 9], rotary, 2, adjacent=adjacent, seed=rotary)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("axes", [0, 1, 2, 3, 4])
@pytest.mark.parametrize("packed", [True, False], ids=["packed", "padded"])
@pytest.mark.parametrize("fused", [True, False], ids=["fused", "apart"])
def test_axes_and_rows(gpu, dtype, axes, packed, fused):
    new = [5, 0, 1, 12, 4] if packed else [4] * 5
    case(gpu, dtype, 8, 2, 64, 16, new, [40, 7, 1, 13, 16], 64, axes, packed=packed, fused=fused, seed=axes, scale=1.25, behind=2 if packed else 0)


@pytest.mark.parametrize("H,H_kv,P", [(1, 1, 8), (28, 4, 16), (32, 32, 1), (8, 8, 256), (128, 16, 16), (5, 1, 32)])
def test_head_layouts_and_pages(gpu, H, H_kv, P):
    for dtype in (BF, F32):
        case(gpu, dtype, H, H_kv, 128, P, [1, 2, 30], [700, 2, 31], 128, 1, seed=H)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_far_positions(gpu, dtype):
    for far in (1 << 22, (1 << 31) - 4000):
        case(gpu, dtype, 4, 2, 64, 16, [7, 3], [50, 3], 64, 3, far=far, seed=4, freqs=np.linspace(1.0, 3.1, 32).astype(np.float32))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rotary,adjacent", [(64, False), (26, False), (64, True), (0, False)])
def test_in_place_append_only_turn_only_and_no_rotation(gpu, dtype, rotary, adjacent):
    for what in ("qk", "q", "k"):
        for in_place in ((False, True) if "q" in what else (False,)):
            case(gpu, dtype, 4, 2, 64, 16, [7, 3], [50, 3], rotary, 1 if rotary else 0, adjacent=adjacent, fused=False, in_place=in_place, what=what,
                 seed=2)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_places_that_do_not_exist_write_nothing(gpu, dtype):
    # more new tokens than the sequence holds: the first ones' places are negative; a sequence without tokens
    w = case(gpu, dtype, 4, 2, 64, 16, [5, 2, 3], [3, 0, 9], 64, 0, seed=3)
    assert w.sum() == 3 + 0 + 3


def test_nothing_to_do(gpu):
    c = Cache(BF, 2, 64, 16, [5], seed=1)
    p, _, _ = c.problem(8)
    gpu.ts_rope_append(p, None, None, None, None, None, 0, None, None)


def test_many_sequences_and_a_long_prompt(gpu):
    rng = np.random.Generator(np.random.PCG64(3))
    lens = rng.integers(0, 9, size=1500).tolist()
    new = [int(rng.integers(0, n + 1)) for n in lens]
    case(gpu, BF, 2, 1, 64, 8, new, lens, 64, 1, seed=9)
    case(gpu, F32, 4, 2, 64, 16, [2500], [3001], 64, 3, seed=10)


def test_a_captured_call_reads_lengths_and_positions_when_it_runs(gpu):
    from paper_2411_02886_amd.runtime import to_device
    c = Cache(BF, 2, 64, 16, [40, 17], seed=1)
    p, kp, vp = c.problem(4)
    rng = np.random.default_rng(0)
    q, k, v = (to_device(W.store(rng.standard_normal((2, h, 64), dtype=np.float32), BF)) for h in (4, 2, 2))
    rope = gpu.Rope(inv_freq=to_device((1e4 ** -(np.arange(32) / 32)).astype(np.float32)))
    pos, lens = to_device(np.array([[9, 12]], np.int32)), p._keep[4]
    out = torch.zeros_like(q)
    k0, v0 = kp.clone(), vp.clone()

    def call(o):
        gpu.ts_rope_append(p, rope, q, k, v, None, 2, pos, o)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        call(out)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        call(out)
    for rep in range(4):
        kp.copy_(k0); vp.copy_(v0); out.zero_()
        torch.cuda.synchronize()
        g.replay(); torch.cuda.synchronize()
        got = [t.clone() for t in (out, kp, vp)]
        kp.copy_(k0); vp.copy_(v0)
        want = torch.zeros_like(out)
        call(want); torch.cuda.synchronize()
        for a, b in zip(got, (want, kp, vp)):
            assert torch.equal(a, b), rep
        pos += 3
        lens -= 1


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("rotary", [4, 8, 12, 20, 28, 36, 40, 56, 72, 100, 120, 124])
def test_parts_that_divide_into_smaller_pieces_or_none(gpu, dtype, adjacent, rotary):
    case(gpu, dtype, 6, 2, 128, 8, [5, 1, 20], [9, 1, 40], rotary, 2, seed=rotary, adjacent=adjacent)
