"""Writing and reading an 8-bit cache with every number of waves to a token that the calls choose among, and the numbers of tokens where the choice changes."""
import pytest

import workloads as W
from test_gpu_quant_cache import case, read

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    return ts


def spread(total):
    """Two sequences that share the tokens, behind others that are there."""
    new = [total - total // 3, total // 3]
    return new, [new[0] + 5, new[1] + 11]


@pytest.mark.parametrize("total", [1, 2, 128, 129, 256, 257, 1024, 1025])
@pytest.mark.parametrize("dtype,code,H,H_kv,D", [(W.BF16, 0, 40, 8, 128), (W.F32, 1, 3, 1, 64)])
def test_tokens_written(gpu, total, dtype, code, H, H_kv, D):
    new, lens = spread(total)
    case(gpu, dtype, code, H, H_kv, D, 16, new, lens, rotary=D, seed=total, behind=2)


# heads that fill the last turn of some waves only, in place and without queries
@pytest.mark.parametrize("H,H_kv", [(1, 1), (2, 1), (5, 1), (6, 2), (28, 4), (32, 4), (128, 32)])
@pytest.mark.parametrize("how", [{}, dict(in_place=True, fused=False), dict(with_q=False)], ids=["", "in place", "no queries"])
def test_heads_that_waves_share(gpu, H, H_kv, how):
    new, lens = spread(7)
    case(gpu, W.BF16, 1, H, H_kv, 128, 8, new, lens, rotary=64, seed=H, **how)


@pytest.mark.parametrize("total", [1, 1024, 1025, 8192, 8193])
@pytest.mark.parametrize("H_kv,D", [(1, 64), (4, 64), (8, 128)])
def test_tokens_read(gpu, total, H_kv, D):
    if total > 1025 and H_kv * D > 256:
        H_kv = 2
    new, lens = spread(total)
    read(gpu, W.BF16, 0, H_kv, D, 16, new, lens, seed=total, behind=1)
