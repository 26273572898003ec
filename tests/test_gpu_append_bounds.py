"""ts_rope_append where lengths lie beyond max_seq_len, as in a captured step that is replayed once too often: such places are not written, places
below the bound are, and angles are those of the true places.  ts_paged_attn takes such a length as max_seq_len."""
import numpy as np
import pytest

import workloads as W
from cache_util import HALF, Cache, attention, check_attention
from test_gpu_rope_append import turned

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


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("rotary", [64, 26, 0])
@pytest.mark.parametrize("packed", [True, False], ids=["packed", "padded"])
@pytest.mark.parametrize("given", [False, True], ids=["", "positions"])
def test_places_beyond_the_bound_are_not_written(gpu, dtype, rotary, packed, given):
    from paper_2411_02886_amd.runtime import to_device, to_host
    H, H_kv, D, P, bound = 4, 2, 64, 8, 16
    new = [1, 3, 30, 5] if packed else [5] * 4
    lens = [17, 9, 40, 18] if packed else [17, 9, 40, 16]          # one past the bound; below; across and wholly beyond
    rng = np.random.Generator(np.random.PCG64(rotary))
    c = Cache(dtype, H_kv, D, P, lens, seed=3)
    p, kp, vp = c.problem(H, chunk=max(new), max_seq_len=bound)
    T, bits = sum(new), dtype == BF
    q, k, v = (W.store(rng.standard_normal((T, h, D), dtype=np.float32), dtype) for h in (H, H_kv, H_kv))
    inv = (1e4 ** -(np.arange(rotary // 2) / max(1, rotary // 2))).astype(np.float32)
    rope = gpu.Rope(inv_freq=to_device(inv)) if rotary else None
    place = np.concatenate([np.arange(N - n, N) for n, N in zip(new, lens)])
    pos = rng.integers(0, 99, (1, T)).astype(np.int32) if given else place[None]
    q_out = to_device(np.zeros_like(q))
    gpu.ts_rope_append(p, rope, to_device(q), to_device(k), to_device(v), to_device(np.cumsum([0] + new).astype(np.int32)) if packed else None, T,
                       to_device(pos) if given else None, q_out)
    torch.cuda.synchronize()
    axes = [0] * (rotary // 2)
    want, tol = turned(W.as_f32(q, dtype).astype(np.float64), pos, inv, axes, False, 1.0)
    err = np.abs(W.as_f32(to_host(q_out, bits16=bits), dtype) - want)
    assert np.all(err <= tol + HALF[dtype] * (np.abs(want) + tol))
    want, tol = turned(W.as_f32(k, dtype).astype(np.float64), pos, inv, axes, False, 1.0)
    kg, vg = (to_host(t, bits16=bits).reshape(-1, H_kv, D) for t in (kp, vp))
    written = np.zeros(len(kg), bool)
    for r, (b, t) in enumerate(zip(np.repeat(np.arange(4), new), place)):
        if t >= bound:
            continue
        s = c.slots(b)[t]
        written[s] = True
        assert np.all(np.abs(W.as_f32(kg[s], dtype) - want[r]) <= (tol + HALF[dtype] * (np.abs(want) + tol))[r]), r
        assert np.array_equal(vg[s], v[r]), r
    assert written.sum() == sum(int(t < bound) for t in place)
    view = np.uint16 if bits else np.uint32
    for now, was in ((kg, c.k_bits), (vg, c.v_bits)):
        assert np.array_equal(np.ascontiguousarray(now[~written]).view(view), np.ascontiguousarray(was[~written]).view(view))


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_a_replayed_step_whose_length_passes_the_bound(gpu, dtype):
    """A captured append of one token per sequence with lengths that grow on the device: the last places keep what the last fitting step wrote."""
    from paper_2411_02886_amd.runtime import to_device, to_host
    H_kv, D, bound = 2, 64, 32
    c = Cache(dtype, H_kv, D, 8, [40, 40], seed=1)
    p, kp, vp = c.problem(4, max_seq_len=bound)
    lens = p._keep[4]
    lens.copy_(torch.tensor([29, 30], dtype=torch.int32))
    rows = to_device(W.store(np.zeros((2, H_kv, D), np.float32), dtype))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(g, stream=side):
        lens += 1
        gpu.ts_rope_append(p, None, None, rows, rows, None, 2, None, None)
    lens.copy_(torch.tensor([29, 30], dtype=torch.int32))
    for step in range(6):
        rows.copy_(to_device(W.store(np.full((2, H_kv, D), step + 1, np.float32), dtype)))
        g.replay()
        torch.cuda.synchronize()
    assert lens.tolist() == [35, 36]
    for t in (kp, vp):
        x = W.as_f32(to_host(t, bits16=dtype == BF).reshape(-1, H_kv, D), dtype)
        assert [float(x[c.slots(0)[i]].max()) for i in (29, 30, 31)] == [1.0, 2.0, 3.0]
        assert [float(x[c.slots(1)[i]].max()) for i in (30, 31)] == [1.0, 2.0]
        was = (c.k if t is kp else c.v)[c.slots(0)]
        assert np.array_equal(x[c.slots(0)[:29]], was[:29]) and np.array_equal(x[c.slots(0)[32:]], was[32:])


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 40])
def test_attention_takes_a_length_beyond_the_bound_as_the_bound(gpu, dtype, n):
    from paper_2411_02886_amd.runtime import to_device, to_host
    c = Cache(dtype, 2, 64, 16, [300, 210], seed=2)
    q = W.store(np.random.default_rng(1).standard_normal((2 * n, 8, 64), dtype=np.float32), dtype)
    p, _, _ = c.problem(8, chunk=n, max_seq_len=200)
    out, lse = to_device(np.zeros_like(q)), torch.zeros((2 * n, 8), device="cuda:0")
    ws = torch.empty((gpu.ts_paged_attn_workspace_bytes(p, 2 * n) + 255) // 256 * 64, dtype=torch.int32, device="cuda:0")
    gpu.ts_paged_attn(p, to_device(q), None, 2 * n, 50, 0.125, out, lse, ws)
    torch.cuda.synchronize()
    c.lens[:] = 200
    check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64),
                    attention(c, q, [n, n], 50, 0.125, [False] * 2), n)
