"""The operators that fill, attend and move a paged cache, as cases that can be timed and compared.

`ts_paged_attn` attends a chunk of new tokens over all of its sequence, `ts_rope_append` turns the new tokens' q and k by
their positions and writes k and v into the pages, `ts_pages_copy` copies pages, `ts_cache_compact` gathers the tokens that
a selection keeps into other pages.  With `own` the library's calls, without it the same from elementary torch
operations.  Inputs are drawn on the GPU from the seed; sequence lengths belong to the case.
"""
import math
import random

import numpy as np
import torch

own = False

_DEV = "cuda:0"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _attn(dtype, B, new, old, H, H_kv, D, P=16, window=0, packed=True, **kw):
    """new, old: (fewest, most) new tokens of a sequence and tokens that its cache holds before them."""
    return dict(op="attn", dtype=dtype, B=B, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1], H=H, H_kv=H_kv, D=D,
                P=P, window=window, packed=packed, **kw)


def _rope(dtype, B, new, old, H, H_kv, D, rotary, axes, P=16, adjacent=False, far=0, **kw):
    """axes: position axes (0: none are given, a token's place in its sequence counts); far: offset of the positions."""
    return dict(op="rope", dtype=dtype, B=B, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1], H=H, H_kv=H_kv, D=D,
                P=P, rotary=rotary, axes=axes, adjacent=adjacent, far=far, **kw)


def _copy(dtype, pages, pool, H_kv, D, P=16, **kw):
    return dict(op="copy", dtype=dtype, pages=pages, pool=pool, H=H_kv, H_kv=H_kv, D=D, P=P, **kw)


def _compact(dtype, B, old, k, n_init, n_local, H, H_kv, D, P=16, **kw):
    return dict(op="compact", dtype=dtype, B=B, new_lo=0, new_hi=0, old_lo=old[0], old_hi=old[1], k=k, n_init=n_init,
                n_local=n_local, H=H, H_kv=H_kv, D=D, P=P, **kw)


def listed():
    return [
        # the smallest layer: one token of one short fp32 sequence, where launches and latency are all there is
        _attn("f32", 1, (1, 1), (4095, 4095), 8, 2, 64, packed=False, name="attn_token_fp32"),
        # a server's batch: one token of each of eight conversations of very different lengths
        _attn("bf16", 8, (1, 1), (16384, 65536), 32, 8, 128, packed=False, name="attn_tokens_batch"),
        # a whole prompt that nothing is cached for
        _attn("bf16", 1, (8192, 8192), (0, 0), 32, 8, 128, packed=False, name="attn_prompt_8k"),
        # a chunk of a long prompt over what its earlier chunks left
        _attn("bf16", 1, (512, 512), (131072, 131072), 32, 8, 128, packed=False, name="attn_chunk_128k"),
        # single tokens beside pieces of prompts, in a layer that sees the last 4096 tokens only (28 heads over 4)
        _attn("bf16", 12, (1, 499), (3, 9001), 28, 4, 128, window=4096, name="attn_mixed_window"),
        # one token of each of a batch
        _rope("bf16", 64, (1, 1), (1000, 30000), 32, 8, 128, 128, 0, name="append_tokens"),
        # pieces of prompts with images and video: time, height and width
        _rope("bf16", 4, (3001, 4500), (0, 5000), 32, 8, 128, 128, 3, name="append_video_prompt"),
        # a part of each head is turned, in fp32, at far positions
        _rope("f32", 3, (1, 777), (5, 4000), 14, 2, 64, 32, 1, adjacent=True, far=1 << 22, name="append_partial_fp32"),
        # eight conversations are forked: the last page of each is copied
        _copy("bf16", 8, 4096, 8, 128, name="copy_fork"),
        # the pages of a pool are moved together
        _copy("bf16", 8000, 20000, 8, 128, name="copy_pool"),
        # conversations whose caches are cut down to what the selection attends
        _compact("bf16", 4, (60000, 131072), 4096, 128, 512, 32, 8, 128, name="compact_128k"),
        # a small fp32 layer's
        _compact("f32", 1, (4096, 4096), 256, 16, 33, 8, 2, 64, name="compact_fp32"),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_one(rng):
    op = rng.choice(["attn", "attn", "attn", "rope", "rope", "copy", "compact"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    H_kv = rng.choice([1, 2, 4, 8, 8, 16])
    H, D, P = H_kv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), rng.choice([64, 128, 128]), rng.choice([8, 16, 16, 32, 64])
    if op == "copy":
        n = _spread(rng, 1, 8000)
        return _copy(dtype, n, 2 * n + rng.randint(1, 4000), H_kv, D, P)
    B = _spread(rng, 1, 32)
    if op == "compact":
        n = _spread(rng, 64, 131072)
        return _compact(dtype, B, (max(1, n // rng.choice([1, 2, 5])), n), _spread(rng, 16, 8192), rng.choice([0, 4, 128]),
                        rng.choice([0, 33, 512]), H, H_kv, D, P)
    if op == "rope":
        B, n = _spread(rng, 1, 256), _spread(rng, 1, 8192)
        return _rope(dtype, B, (max(1, n // rng.choice([1, 3, 50])), n), (rng.choice([0, 7]), _spread(rng, 8, 20000)), H, H_kv, D,
                     rng.choice([D, D, D // 2, 24]), rng.choice([0, 0, 1, 2, 3, 4]), P, rng.choice([False, True]),
                     rng.choice([0, 0, 1 << 20]))
    n = rng.choice([1, 1, _spread(rng, 2, 8), _spread(rng, 9, 8192)])
    old = _spread(rng, 1, 131072)
    return _attn(dtype, B, (n if rng.random() < 0.5 else 1, n), (rng.choice([0, old // 4, old]), old), H, H_kv, D, P,
                 rng.choice([0, 0, 0, 1024, 4096]), rng.random() < 0.5)


def draw(rng):
    big = _attn("bf16", 1, (512, 512), (131072, 131072), 32, 8, 128)
    top = max(work(c)["flops"] for c in listed())
    while True:
        c = _draw_one(rng)
        if c["H"] > 128 or (c["op"] != "copy" and _tokens(c) * _row(c) > 1 << 31):
            continue
        if c["op"] == "attn" and not c["packed"]:
            c["new_lo"] = c["new_hi"]       # [B][C][H][D]: every sequence has as many
        w = work(c)
        if w["flops"] > top or w["bytes"] > 4e9 or w["bytes"] < 1e5:
            continue
        if c["op"] == "attn":
            scores = c["B"] * c["H"] * c["new_hi"] * (c["new_hi"] + c["old_hi"])
            if scores > 32 * 512 * 131584 or (c["dtype"] == "f32" and w["flops"] > work(big)["flops"] / 16):
                continue                    # products in 32 bits have a sixteenth of the rate
        return c


# ---------------------------------------------------------------------------------------------------------------------
# sizes

def _lengths(c):
    """(new tokens, tokens before them) of every sequence: the case's own."""
    rng = random.Random("%(B)d %(new_lo)d %(new_hi)d %(old_lo)d %(old_hi)d %(H)d %(H_kv)d %(D)d" % c)
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(c["B"])]
    old = [rng.randint(c["old_lo"], c["old_hi"]) for _ in range(c["B"])]
    new[0], old[-1] = c["new_hi"], c["old_hi"]
    return new, old


def _tokens(c):
    new, old = _lengths(c)
    return sum(new) + sum(old)


def _row(c):
    """Bytes of a token's K (or V)."""
    return c["H_kv"] * c["D"] * _BYTES[c["dtype"]]


def _kept(c):
    """Tokens that a compaction keeps of every sequence."""
    kept = []
    for n in _lengths(c)[1]:
        lo = min(c["n_init"], n)
        hi = max(lo, n - c["n_local"])
        kept.append((lo, min(c["k"], hi - lo), hi, n))
    return kept


def work(case):
    c, es = case, _BYTES[case["dtype"]]
    if c["op"] == "copy":
        return dict(bytes=4 * c["pages"] * c["P"] * _row(c) + 8 * c["pages"], flops=0)
    if c["op"] == "compact":
        kept = sum(lo + m + n - hi for lo, m, hi, n in _kept(c))
        return dict(bytes=4 * kept * _row(c) + 4 * sum(m for _, m, _, _ in _kept(c)), flops=0)
    new, old = _lengths(c)
    T = sum(new)
    if c["op"] == "rope":
        return dict(bytes=2 * T * (c["H"] * c["D"] * es + 2 * _row(c)) + 4 * T * c["axes"],
                    flops=3.0 * T * (c["H"] + c["H_kv"]) * c["rotary"])
    pairs, cached = 0, 0
    for n, o in zip(new, old):
        w = c["window"] if c["window"] else n + o
        first = min(n, max(0, w - o))       # rows that the window does not cut
        pairs += first * o + first * (first + 1) // 2 + (n - first) * w
        cached += min(n + o, w + n - 1)
    return dict(bytes=2 * cached * _row(c) + 2 * T * c["H"] * c["D"] * es + 4 * T * c["H"], flops=4.0 * pairs * c["H"] * c["D"])


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _gen(seed, salt=0):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + salt)


def _pools(c, pages, g):
    tdt = _TORCH[c["dtype"]]
    return [torch.randn((pages, c["P"], c["H_kv"], c["D"]), generator=g, device=_DEV, dtype=torch.float32).to(tdt) for _ in "kv"]


def _int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=_DEV)


def _inputs(c, seed):
    """What every pass of a case starts from; nothing in it depends on how the pass is computed."""
    g, P, D, H, H_kv, tdt = _gen(seed), c["P"], c["D"], c["H"], c["H_kv"], _TORCH[c["dtype"]]
    x = {}
    if c["op"] == "copy":
        x["k_pool"], x["v_pool"] = _pools(c, c["pool"], g)
        perm = torch.randperm(c["pool"], generator=g, device=_DEV).int()
        x["src"], x["dst"] = perm[:c["pages"]].contiguous(), perm[c["pages"]:2 * c["pages"]].contiguous()
        x["lens"], x["indptr"], x["pages"] = _int32([P]), _int32([0, 1]), _int32([0])
        x["max_len"], x["new"] = P, 1
        return x
    new, old = _lengths(c)
    T, lens = sum(new), [n + o for n, o in zip(new, old)]
    need = [(n + P - 1) // P for n in lens]
    kept = [(lo + m + n - hi + P - 1) // P for lo, m, hi, n in _kept(c)] if c["op"] == "compact" else []
    perm = torch.randperm(sum(need) + sum(kept) + 3, generator=g, device=_DEV).int()
    x["k_pool"], x["v_pool"] = _pools(c, perm.numel(), g)
    x["indptr"], x["pages"] = _int32(np.cumsum([0] + need)), perm[:sum(need)].contiguous()
    x["lens"], x["max_len"] = _int32(lens), max(lens)
    x["q_indptr"], x["new"] = _int32(np.cumsum([0] + new)), max(new)
    if c["op"] == "compact":
        x["to_indptr"], x["to_pages"] = _int32(np.cumsum([0] + kept)), perm[sum(need):sum(need) + sum(kept)].contiguous()
        x["to_lens"] = torch.zeros((c["B"],), dtype=torch.int32, device=_DEV)
        x["idx"] = torch.full((c["B"], c["k"]), -1, dtype=torch.int32, device=_DEV)
        for b, (lo, m, hi, n) in enumerate(_kept(c)):
            x["idx"][b, :m] = (lo + torch.randperm(hi - lo, generator=g, device=_DEV)[:m].sort().values).int()
        x["count"] = _int32([m for _, m, _, _ in _kept(c)])
        return x
    if c["op"] == "rope":
        # one projection's output: q, k and v of a token follow each other
        qkv = torch.randn((T, (H + 2 * H_kv) * D), generator=g, device=_DEV).to(tdt)
        x["q"], x["k"], x["v"] = qkv[:, :H * D], qkv[:, H * D:(H + H_kv) * D], qkv[:, (H + H_kv) * D:]
        half = c["rotary"] // 2
        x["inv_freq"] = (1e6 ** -(torch.arange(half, device=_DEV, dtype=torch.float64) / half)).float()
        n_ax = max(1, c["axes"])
        x["pair_axis"] = [i % n_ax for i in range(half)]
        x["positions"] = None
        if c["axes"]:
            x["positions"] = (torch.randint(0, 40000, (c["axes"], T), generator=g, device=_DEV) + c["far"]).int()
        return x
    # queries lean towards a direction that the first tokens' keys share: the logits of those stand out
    lean = torch.randn((H_kv, D), generator=g, device=_DEV)
    lean = 8.0 * lean / lean.norm(dim=-1, keepdim=True)
    x["q"] = (torch.randn((T, H, D), generator=g, device=_DEV) + lean.repeat_interleave(H // H_kv, dim=0)).to(tdt)
    first = [(int(a) * P + np.arange(min(4, n))) for a, n in zip(np.cumsum([0] + need)[:-1], lens)]
    t = torch.tensor(np.concatenate(first), device=_DEV)
    slot = x["pages"][t // P].long() * P + t % P
    flat = x["k_pool"].view(-1, H_kv, D)
    flat[slot] = (flat[slot].float() + lean).to(tdt)
    return x


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    s = dict(c=c, x=x, sm=1.0 / math.sqrt(c["D"]))
    tdt = _TORCH[c["dtype"]]
    if c["op"] == "attn":
        T = x["q"].shape[0]
        s["out"] = torch.zeros((T, c["H"], c["D"]), dtype=tdt, device=_DEV)
        s["lse"] = torch.zeros((T, c["H"]), dtype=torch.float32, device=_DEV)
    if c["op"] == "rope":
        s["q_out"] = torch.zeros((x["q"].shape[0], c["H"], c["D"]), dtype=tdt, device=_DEV)
    if own:     # the handle of the layer's cache, the rotation and the workspace, which a program keeps
        from paper_2411_02886_amd import binding as ts
        s["ts"] = ts
        s["problem"] = ts.Problem(batch=c.get("B", 1), chunk=x["new"] or 1, num_q_heads=c["H"], num_kv_heads=c["H_kv"],
                                  head_dim=c["D"], page_size=c["P"], max_seq_len=x["max_len"],
                                  dtype=ts.TS_BF16 if c["dtype"] == "bf16" else ts.TS_F32, k_pool=x["k_pool"], v_pool=x["v_pool"],
                                  page_indptr=x["indptr"], page_indices=x["pages"], seq_lens=x["lens"],
                                  num_initial=c.get("n_init", 0), num_local=c.get("n_local", 0))
        if c["op"] == "attn":
            n = ts.ts_paged_attn_workspace_bytes(s["problem"], x["q"].shape[0])
            s["ws"] = torch.empty(((n + 255) // 256 * 64,), dtype=torch.int32, device=_DEV)
        if c["op"] == "rope":
            s["rope"] = ts.Rope(inv_freq=x["inv_freq"], pair_axis=x["pair_axis"], num_axes=max(1, c["axes"]),
                                adjacent=c["adjacent"])
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass

def _run_own(s):
    c, x, ts = s["c"], s["x"], s["ts"]
    if c["op"] == "attn":
        ts.ts_paged_attn(s["problem"], x["q"], x["q_indptr"] if c["packed"] else None, x["q"].shape[0], c["window"], s["sm"],
                         s["out"], s["lse"], s["ws"])
        return dict(out=s["out"], lse=s["lse"])
    if c["op"] == "rope":
        ts.ts_rope_append(s["problem"], s["rope"], x["q"], x["k"], x["v"], x["q_indptr"], x["q"].shape[0], x["positions"],
                          s["q_out"])
        return dict(q=s["q_out"], k_pool=x["k_pool"], v_pool=x["v_pool"])
    if c["op"] == "copy":
        ts.ts_pages_copy(s["problem"], x["src"], x["dst"], c["pages"], c["pool"])
        return dict(k_pool=x["k_pool"], v_pool=x["v_pool"])
    ts.ts_cache_compact(s["problem"], x["idx"], c["k"], x["count"], None, x["to_indptr"], x["to_pages"], x["to_lens"])
    return dict(k_pool=x["k_pool"], v_pool=x["v_pool"], lens=x["to_lens"])


def _slots(indptr, pages, t, P):
    """Rows of the pool, [B][len(t)], of logical tokens t [len] or [B][len]; those that do not exist read some page."""
    at = indptr[:-1, None].long() + (t // P if t.dim() == 2 else (t // P)[None, :])
    return pages[at.clamp(max=pages.numel() - 1)].long() * P + t % P


def _plain_attn(s):
    c, x = s["c"], s["x"]
    B, H, H_kv, D, P, T = c["B"], c["H"], c["H_kv"], c["D"], c["P"], x["q"].shape[0]
    G, C, N = H // H_kv, x["new"], x["max_len"]
    start = x["q_indptr"][:-1].long()
    new = x["q_indptr"][1:].long() - start
    chunk, t = torch.arange(C, device=_DEV), torch.arange(N, device=_DEV)
    q = x["q"][(start[:, None] + chunk).clamp(max=T - 1)].float()                       # [B][C][H][D]
    q = q.view(B, C, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(B * H_kv, C * G, D)
    slot = _slots(x["indptr"], x["pages"], t, P)
    k = x["k_pool"].view(-1, H_kv, D)[slot].float().permute(0, 2, 3, 1).reshape(B * H_kv, D, N)
    pos = x["lens"].long()[:, None] - new[:, None] + chunk                              # [B][C]
    seen = t[None, None, :] <= pos[:, :, None]
    if c["window"]:
        seen &= t[None, None, :] > pos[:, :, None] - c["window"]
    logits = torch.bmm(q, k).view(B, H_kv, C, G, N).mul_(s["sm"])
    del k
    logits.masked_fill_(~seen[:, None, :, None, :], -math.inf)
    top = logits.amax(dim=-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    weights = logits.sub_(top).exp_()
    total = weights.sum(dim=-1, keepdim=True)
    v = x["v_pool"].view(-1, H_kv, D)[slot].float().permute(0, 2, 1, 3).reshape(B * H_kv, N, D)
    o = torch.bmm(weights.view(B * H_kv, C * G, N), v).view(B, H_kv, C, G, D) / total.clamp(min=1e-38)
    lse = (top + total.log())[..., 0]
    row = torch.arange(T, device=_DEV)
    b = torch.bucketize(row, x["q_indptr"][1:].long(), right=True)
    at = row - start[b]
    o = o.permute(0, 2, 1, 3, 4).reshape(B, C, H, D)[b, at]
    lse = lse.permute(0, 2, 1, 3).reshape(B, C, H)[b, at]
    return dict(out=o.to(s["out"].dtype), lse=lse)


def _row_places(x, P):
    """(sequence's place in its pages, pool row) of every new token: [T]."""
    row = torch.arange(x["q"].shape[0], device=_DEV)
    end = x["q_indptr"][1:].long()
    b = torch.bucketize(row, end, right=True)
    t = x["lens"].long()[b] - end[b] + row
    return t, x["pages"][x["indptr"][b].long() + t // P].long() * P + t % P


def _angles(c, x, t):
    """[T][pairs] in 64 bits: of far positions the angle in 32 bits has no fraction left."""
    pos = x["positions"] if x["positions"] is not None else t[None, :]
    axis = torch.tensor(x["pair_axis"], device=_DEV)
    return pos[axis].t().double() * x["inv_freq"].double()


def _turn(c, rows, cos, sin):
    """rows [T][heads][D] turned pair by pair; what lies behind the rotated part stays."""
    r = c["rotary"]
    if c["adjacent"]:
        a, b = rows[..., 0:r:2], rows[..., 1:r:2]
    else:
        a, b = rows[..., :r // 2], rows[..., r // 2:r]
    cos, sin = cos[:, None, :], sin[:, None, :]
    ra, rb = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack((ra, rb), dim=-1).flatten(-2) if c["adjacent"] else torch.cat((ra, rb), dim=-1)
    return torch.cat((turned, rows[..., r:]), dim=-1)


def _plain_rope(s):
    c, x = s["c"], s["x"]
    T, tdt = x["q"].shape[0], s["q_out"].dtype
    t, slot = _row_places(x, c["P"])
    angle = _angles(c, x, t)
    cos, sin = angle.cos().float(), angle.sin().float()
    q = _turn(c, x["q"].view(T, c["H"], c["D"]).float(), cos, sin).to(tdt)
    k = _turn(c, x["k"].view(T, c["H_kv"], c["D"]).float(), cos, sin).to(tdt)
    x["k_pool"].view(-1, c["H_kv"], c["D"])[slot] = k
    x["v_pool"].view(-1, c["H_kv"], c["D"])[slot] = x["v"].view(T, c["H_kv"], c["D"])
    return dict(q=q, k_pool=x["k_pool"], v_pool=x["v_pool"])


def _plain_copy(s):
    x = s["x"]
    src, dst = x["src"].long(), x["dst"].long()
    x["k_pool"][dst] = x["k_pool"][src]
    x["v_pool"][dst] = x["v_pool"][src]
    return dict(k_pool=x["k_pool"], v_pool=x["v_pool"])


def _plain_compact(s):
    c, x = s["c"], s["x"]
    n = x["lens"].long()[:, None]
    lo = n.clamp(max=c["n_init"])
    hi = torch.maximum(lo, n - c["n_local"])
    count = x["count"].long()[:, None]
    j = torch.arange(c["n_init"] + c["k"] + c["n_local"], device=_DEV)[None, :]
    chosen = x["idx"].long().gather(1, (j - lo).clamp(min=0, max=c["k"] - 1))
    total = lo + count + n - hi
    token = torch.where(j < lo, j, torch.where(j < lo + count, chosen, hi + j - lo - count))
    token, j = torch.where(j < total, token, token[:, :1]), torch.where(j < total, j, 0)    # past the end: the first again
    src, dst = _slots(x["indptr"], x["pages"], token, c["P"]), _slots(x["to_indptr"], x["to_pages"], j, c["P"])
    for pool in (x["k_pool"].view(-1, c["H_kv"], c["D"]), x["v_pool"].view(-1, c["H_kv"], c["D"])):
        pool[dst] = pool[src]
    x["to_lens"].copy_(total[:, 0])
    return dict(k_pool=x["k_pool"], v_pool=x["v_pool"], lens=x["to_lens"])


def run(state):
    if own:
        return _run_own(state)
    return {"attn": _plain_attn, "rope": _plain_rope, "copy": _plain_copy, "compact": _plain_compact}[state["c"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence

def _exact_attn(c, x):
    T, H, D, P, H_kv = x["q"].shape[0], c["H"], c["D"], c["P"], c["H_kv"]
    G = H // H_kv
    out = torch.zeros((T, H, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=_DEV)
    new, old = _lengths(c)
    pages, first, row = x["pages"].long(), x["indptr"].tolist(), 0
    for b, (n, o) in enumerate(zip(new, old)):
        N = n + o
        t = torch.arange(N, device=_DEV)
        slot = pages[first[b] + t // P] * P + t % P
        step = max(1, (1 << 28) // max(1, N * G))
        for kv in range(H_kv):
            k, v = (x[p].view(-1, H_kv, D)[slot, kv].double() for p in ("k_pool", "v_pool"))
            for a in range(0, n, step):
                m = min(step, n - a)
                qs = x["q"][row + a:row + a + m, kv * G:(kv + 1) * G].double().reshape(m * G, D)
                z = (qs @ k.t().contiguous() / math.sqrt(D)).view(m, G, N)
                at = o + a + torch.arange(m, device=_DEV)[:, None]
                hidden = t[None, :] > at
                if c["window"]:
                    hidden |= t[None, :] <= at - c["window"]
                z.masked_fill_(hidden[:, None, :], -math.inf)
                l = torch.logsumexp(z, dim=-1)
                out[row + a:row + a + m, kv * G:(kv + 1) * G] = (torch.exp(z - l[..., None]).view(m * G, N) @ v).view(m, G, D)
                lse[row + a:row + a + m, kv * G:(kv + 1) * G] = l
        row += n
    return dict(out=out, lse=lse)


def _exact_rope(c, x):
    new, old = _lengths(c)
    H, H_kv, D, P = c["H"], c["H_kv"], c["D"], c["P"]
    kp, vp = (x[p].double().view(-1, H_kv, D) for p in ("k_pool", "v_pool"))
    q, k, v = (x[n].double().view(-1, h, D).clone() for n, h in (("q", H), ("k", H_kv), ("v", H_kv)))
    place = torch.cat([torch.arange(o, o + n, device=_DEV) for n, o in zip(new, old)])
    page = torch.cat([x["pages"].long()[int(a) + torch.arange(o, o + n, device=_DEV) // P]
                      for a, n, o in zip(x["indptr"].tolist(), new, old)])
    for i in range(c["rotary"] // 2):
        pos = place if x["positions"] is None else x["positions"][x["pair_axis"][i]].long()
        z = torch.polar(torch.ones_like(pos, dtype=torch.float64), pos.double() * float(x["inv_freq"][i]))[:, None]
        e0, e1 = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + c["rotary"] // 2)
        for rows in (q, k):
            w = torch.complex(rows[..., e0], rows[..., e1]) * z
            rows[..., e0], rows[..., e1] = w.real, w.imag
    kp[page * P + place % P] = k
    vp[page * P + place % P] = v
    shape = x["k_pool"].shape
    return dict(q=q, k_pool=kp.view(shape), v_pool=vp.view(shape))


def exact(case, seed):
    c, x = case, _inputs(case, seed)
    if c["op"] == "attn":
        return _exact_attn(c, x)
    if c["op"] == "rope":
        return _exact_rope(c, x)
    shape = x["k_pool"].shape
    if c["op"] == "copy":
        to = torch.arange(c["pool"], device=_DEV)
        to[x["dst"].long()] = x["src"].long()           # where each page's contents come from
        return dict(k_pool=x["k_pool"][to].double(), v_pool=x["v_pool"][to].double())
    to, lens = torch.arange(shape[0] * c["P"], device=_DEV), []
    for b, (lo, m, hi, n) in enumerate(_kept(c)):
        t = torch.cat([torch.arange(lo, device=_DEV), x["idx"][b, :m].long(), torch.arange(hi, n, device=_DEV)])
        j = torch.arange(t.numel(), device=_DEV)
        at = [pages.long()[int(ptr[b]) + i // c["P"]] * c["P"] + i % c["P"]
              for ptr, pages, i in ((x["to_indptr"], x["to_pages"], j), (x["indptr"], x["pages"], t))]
        to[at[0]] = at[1]
        lens.append(t.numel())
    k, v = (x[p].view(-1, c["H_kv"], c["D"])[to].double().view(shape) for p in ("k_pool", "v_pool"))
    return dict(k_pool=k, v_pool=v, lens=_int32(lens))
