"""What the binding of the cache's calls refuses before anything is launched: tensors whose layout or type the library cannot see."""
import pytest

import paper_2411_02886_amd as ts

torch = pytest.importorskip("torch")


def problem(dtype=None, **kw):
    z = torch.zeros(4, dtype=torch.int32)
    args = dict(batch=1, num_q_heads=4, num_kv_heads=2, head_dim=64, page_size=16, max_seq_len=9, dtype=ts.TS_F32 if dtype is None else dtype,
                k_pool=z, v_pool=z, page_indptr=z, page_indices=z, seq_lens=z)
    args.update(kw)
    return ts.Problem(**args)


@pytest.mark.parametrize("what", ["q", "k", "v"])
def test_rows_that_overlap_are_refused(what):
    """Stride 0 would be taken as packed: rows would be read behind the one that is there."""
    ind = torch.zeros(2, dtype=torch.int32)
    heads = dict(q=4, k=2, v=2)
    for shape in ((3, heads[what], 64), (3, heads[what] * 64)):
        a = {n: torch.zeros(3, h, 64) for n, h in heads.items()}
        for bad in (torch.zeros(1, *shape[1:]).expand(*shape), torch.zeros(3 * 64 * 8).as_strided(shape, (64,) + ((64, 1) if len(shape) == 3 else (1,)))):
            a[what] = bad
            with pytest.raises(ValueError):
                ts.ts_rope_append(problem(), None, a["q"], a["k"], a["v"], ind, 3, None, torch.zeros(3, 4, 64))
