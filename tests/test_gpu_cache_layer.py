"""The cache's calls as the layers offer them: lists of copies, shapes, workspaces, streams."""
import numpy as np
import pytest

import workloads as W
from cache_util import Cache, attention, check_attention

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


def test_joined_lists_of_page_copies_are_made_in_their_order(gpu):
    from paper_2411_02886_amd.pages import PagePool
    from paper_2411_02886_amd.runtime import copy_pages
    P, NP = 256, 64
    k = torch.arange(NP, dtype=torch.int32, device="cuda:0")[:, None, None, None].repeat(1, P, 2, 64)
    v = -k
    z = torch.zeros(4, dtype=torch.int32, device="cuda:0")
    p = gpu.Problem(batch=1, num_q_heads=2, num_kv_heads=2, head_dim=64, page_size=P, max_seq_len=1, dtype=F32, k_pool=k, v_pool=v, page_indptr=z,
                    page_indices=z, seq_lens=z)
    pool, copies = PagePool(NP, P), []
    pool.add(0, 3)
    for i in range(NP - 1):                              # each child forks the one before and grows: a chain of copies
        pool.fork(i, i + 1)
        copies += pool.grow(i + 1)
    assert copies == [(i, i + 1) for i in range(NP - 1)]
    copy_pages(p, copies, NP)
    torch.cuda.synchronize()
    assert not k.any() and not v.any()


def test_two_streams_attend_on_one_layer(gpu):
    from paper_2411_02886_amd.runtime import DecodeLayer, to_device, to_host
    c = Cache(BF, 2, 64, 16, [9000, 4000, 2500], seed=8)
    lay = DecodeLayer(dtype=BF, H=8, H_kv=2, D=64, P=16, k=16, k_pool=c.k_bits.reshape(-1, 16, 2, 64), v_pool=c.v_bits.reshape(-1, 16, 2, 64),
                      page_indptr=c.indptr, page_indices=c.pages, seq_lens=c.lens)
    rng = np.random.default_rng(1)
    q = [W.store(rng.standard_normal((3, 8, 64), dtype=np.float32), BF) for _ in range(2)]
    dev = [to_device(x) for x in q]
    got = [(torch.zeros((3, 8, 64), dtype=torch.int16, device="cuda:0"), torch.zeros((3, 8), device="cuda:0")) for _ in range(2)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for rep in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                lay.attend_all(dev[i], out=got[i][0], lse=got[i][1])
    torch.cuda.synchronize()
    assert len({w.data_ptr() for w in lay._all_ws.values()}) == 2
    for i in range(2):
        check_attention(W.as_f32(to_host(got[i][0], bits16=True), BF).astype(np.float64), to_host(got[i][1]).astype(np.float64),
                        attention(c, q[i], [1] * 3, 0, 0.125, [False] * 3), i)


def test_a_chunk_is_appended_and_attended_in_one_shape(gpu):
    """[B][C][heads][D] parts of a projection, for append and attend_all alike."""
    from paper_2411_02886_amd.runtime import ChunkSelector, to_device, to_host
    B, C, H, H_kv, D, P = 2, 20, 8, 2, 64, 16
    c = Cache(BF, H_kv, D, P, [70, 33], seed=8)
    x = W.store(np.random.default_rng(2).standard_normal((B, C, H + 2 * H_kv, D), dtype=np.float32), BF)
    for b in range(B):
        at = c.slots(b)[-C:]
        for bits, now, part in ((c.k_bits, c.k, x[b, :, H:H + H_kv]), (c.v_bits, c.v, x[b, :, H + H_kv:])):
            now[at] = W.as_f32(part, BF)
    sel = ChunkSelector(C=C, H=H, H_kv=H_kv, D=D, P=P, k=8, k_pool=c.k_bits.reshape(-1, P, H_kv, D), v_pool=c.v_bits.reshape(-1, P, H_kv, D),
                        page_indptr=c.indptr, page_indices=c.pages, seq_lens=c.lens)
    dev = to_device(x)
    q = torch.zeros((B, C, H, D), dtype=torch.int16, device="cuda:0")
    sel.append(dev[:, :, H:H + H_kv], dev[:, :, H + H_kv:], q=dev[:, :, :H], q_out=q)
    sel.attend_all(q)
    torch.cuda.synchronize()
    check_attention(W.as_f32(to_host(sel.out, bits16=True), BF).astype(np.float64).reshape(B * C, H, D), to_host(sel.lse).astype(np.float64).reshape(B * C, H),
                    attention(c, x[:, :, :H].reshape(B * C, H, D), [C, C], 0, 0.125, [False] * 2), "chunk")


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
def test_prompts_on_a_decode_layer(gpu, dtype):
    """Packed prompts with and without a bound on their lengths."""
    from paper_2411_02886_amd.runtime import DecodeLayer, to_device, to_host
    c = Cache(dtype, 2, 64, 16, [900, 400, 250], seed=8)
    lay = DecodeLayer(dtype=dtype, H=8, H_kv=2, D=64, P=16, k=16, k_pool=c.k_bits.reshape(-1, 16, 2, 64), v_pool=c.v_bits.reshape(-1, 16, 2, 64),
                      page_indptr=c.indptr, page_indices=c.pages, seq_lens=c.lens)
    new = [300, 1, 60]
    q = W.store(np.random.default_rng(1).standard_normal((361, 8, 64), dtype=np.float32), dtype)
    ref = attention(c, q, new, 0, 0.125, [False] * 3)
    out, lse, ind = to_device(np.zeros_like(q)), torch.zeros((361, 8), device="cuda:0"), to_device(np.cumsum([0] + new).astype(np.int32))
    for most in (None, 300, 1000, 2):
        out.zero_(), lse.zero_()
        lay.attend_all(to_device(q), q_indptr=ind, out=out, lse=lse, most_new=most)
        torch.cuda.synchronize()
        check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64), to_host(lse).astype(np.float64), ref, most)


@pytest.mark.parametrize("dtype", [BF, F32], ids=["bf16", "f32"])
@pytest.mark.parametrize("new", [[1, 3, 0, 2], [40, 1, 0, 90], [300, 5, 200, 1]])
@pytest.mark.parametrize("B", [4, 70])
def test_rows_in_front_of_the_first_sequence_and_behind_the_last(gpu, dtype, new, B):
    """q_indptr may begin above 0: those rows are nobody's, as are the ones behind its end."""
    from paper_2411_02886_amd.runtime import to_device, to_host
    H, H_kv, D, front, behind = 8, 2, 64, 7, 5
    new = new + [1, 0] * ((B - 4) // 2)
    lens = [n + 11 * (b % 5) for b, n in enumerate(new)]
    c = Cache(dtype, H_kv, D, 16, lens, seed=B)
    T = front + sum(new) + behind
    x = W.store(np.random.default_rng(2).standard_normal((T, H + 2 * H_kv, D), dtype=np.float32), dtype)
    mine = slice(front, T - behind)
    ind = to_device((front + np.cumsum([0] + new)).astype(np.int32))
    for b in range(B):
        at, r = c.slots(b)[lens[b] - new[b]:], front + sum(new[:b])
        for bits, now, part in ((c.k_bits, c.k, x[r:r + new[b], H:H + H_kv]), (c.v_bits, c.v, x[r:r + new[b], H + H_kv:])):
            now[at] = W.as_f32(part, dtype)
    for bound in (None, 1 << 20):
        p, kp, vp = c.problem(H, chunk=max(new), max_seq_len=bound)
        dev = to_device(x)
        q_out, out = (torch.full((T, H, D), 7, dtype=dev.dtype, device="cuda:0") for _ in "ab")
        lse = torch.full((T, H), 7.0, device="cuda:0")
        gpu.ts_rope_append(p, None, dev[:, :H], dev[:, H:H + H_kv], dev[:, H + H_kv:], ind, T, None, q_out)
        ws = torch.empty((gpu.ts_paged_attn_workspace_bytes(p, T) + 255) // 256 * 64, dtype=torch.int32, device="cuda:0")
        gpu.ts_paged_attn(p, q_out, ind, T, 0, 0.125, out, lse, ws)
        torch.cuda.synchronize()
        nobody = np.r_[0:front, T - behind:T]
        assert all(np.all(to_host(t)[nobody] == 7) for t in (q_out, out, lse))
        ref = attention(c, x[mine, :H], new, 0, 0.125, [False] * B)
        check_attention(W.as_f32(to_host(out, bits16=dtype == BF), dtype).astype(np.float64)[mine], to_host(lse).astype(np.float64)[mine], ref, bound)
        for t, want in ((kp, c.k), (vp, c.v)):
            got = W.as_f32(to_host(t, bits16=dtype == BF).reshape(want.shape), dtype)
            assert np.array_equal(np.isnan(got), np.isnan(want)) and np.array_equal(got[~np.isnan(got)], want[~np.isnan(want)].astype(np.float32))
