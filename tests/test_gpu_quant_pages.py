"""ts_quant_pages_copy of as many pages as a server moves at once: more than a launch has workgroups, of every size of page, in pools beyond 4 GiB."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2411_02886_amd as ts
    ts.load()
    yield ts
    torch.cuda.empty_cache()


@pytest.mark.parametrize("pages,copies,P,H_kv,D", [(50000, 20000, 8, 1, 64), (40001, 20000, 16, 2, 64), (9000, 4096, 16, 8, 128), (70000, 33000, 4, 2, 128),
                                                   (17000, 8000, 64, 32, 128)])       # (the last: 4.1 GiB of codes each)
def test_many_pages(gpu, pages, copies, P, H_kv, D):
    g = torch.Generator(device="cuda:0").manual_seed(pages)
    cache = gpu.QuantCache.empty(pages, P, H_kv, D, gpu.TS_INT8)
    for t in cache._keep:
        if t.dtype == torch.uint8:
            t.random_(0, 256, generator=g)
        else:
            t.normal_(generator=g)
    z = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    p = gpu.Problem(batch=1, num_q_heads=H_kv, num_kv_heads=H_kv, head_dim=D, page_size=P, max_seq_len=1, dtype=gpu.TS_BF16, k_pool=None, v_pool=None,
                    page_indptr=z, page_indices=z, seq_lens=z)
    perm = torch.randperm(pages, generator=g, device="cuda:0")
    src, dst = perm[:copies], perm[copies:2 * copies]
    src = src[torch.randint(0, copies, (dst.numel(),), generator=g, device="cuda:0")]       # some pages go to several places
    want = [t.clone() for t in cache._keep]
    for t in want:
        t[dst] = t[src]
    gpu.ts_quant_pages_copy(p, cache, src.int(), dst.int(), dst.numel(), pages)
    torch.cuda.synchronize()
    for name, a, b in zip(("k_codes", "v_codes", "k_scale", "v_scale"), cache._keep, want):
        assert torch.equal(a, b), name
