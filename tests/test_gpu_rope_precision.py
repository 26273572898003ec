"""ts_rope_append, fp32: sine and cosine are rounded once, from 64 bits."""
import numpy as np
import pytest

import workloads as W
from cache_util import Cache

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = W.F32


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


@pytest.mark.parametrize("adjacent", [False, True], ids=["halves", "neighbours"])
@pytest.mark.parametrize("rotary", [26, 64])
@pytest.mark.parametrize("scale", [1.0, 1.25, -0.7])
def test_sine_and_cosine_are_half_a_step_off_at_most(gpu, adjacent, rotary, scale):
    """Unit pairs (1, 0) come out as scale * (cos, sin): one rounding, 2^-24 of the value, beside the angle's own in 64 bits (two roundings of it, 2^-52)
    and that of functions and factor (2^-50)."""
    from paper_2411_02886_amd.runtime import to_device, to_host
    T, H, D, half = 3000, 1, 64, rotary // 2
    rng = np.random.Generator(np.random.PCG64(rotary))
    pos = np.concatenate([np.arange(1000), rng.integers(-70000, 200000, T - 1000)]).astype(np.int32)
    inv = (1e4 ** -(np.arange(half) / half)).astype(np.float32)
    x = np.zeros((T, H, D), np.float32)
    e0, e1 = (2 * np.arange(half), 2 * np.arange(half) + 1) if adjacent else (np.arange(half), np.arange(half) + half)
    x[..., e0] = 1.0
    c = Cache(F32, 1, D, 16, [T], seed=1)
    p, _, _ = c.problem(H, chunk=T)
    out = torch.zeros((T, H, D), device="cuda:0")
    gpu.ts_rope_append(p, gpu.Rope(inv_freq=to_device(inv), adjacent=adjacent, scale=scale), to_device(x), None, None, None, T, to_device(pos[None]), out)
    torch.cuda.synchronize()
    got = to_host(out).astype(np.float64)[:, 0]
    a, sc = pos.astype(np.float64)[:, None] * inv.astype(np.float64)[None], float(np.float32(scale))
    for e, f in ((e0, np.cos), (e1, np.sin)):
        want = sc * f(a)
        assert np.all(np.abs(got[:, e] - want) <= np.abs(want) * 2.0 ** -24 + abs(sc) * (np.abs(a) * 2.0 ** -51 + 2.0 ** -50))
