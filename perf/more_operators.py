"""The operators of an 8-bit paged cache and of drafted trees, as cases that can be timed and compared.

`ts_quant_append` writes new tokens into pages of 8-bit codes, `ts_quant_read` reads tokens back, `ts_quant_attn` attends
over such a cache; `ts_tree_mask` says which drafted tokens of a tree see which, `ts_tree_attn` (or `ts_quant_attn` with the
mask) attends with it, `ts_tree_keep` closes up the rows of the accepted path.  With `own` the library's calls, without it the
same from elementary torch operations.  Inputs are drawn on the GPU from the seed; sequence lengths belong to the case.
"""
import math
import random

import numpy as np
import torch

own = False

_DEV = "cuda:0"
_TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}
_TOP = {"int8": 127.0, "e4m3": 448.0}       # the largest code


def _case(op, dtype, fmt, B, new, old, H, H_kv, D, P=16, window=0, packed=True, rotary=0, adjacent=False, most_kept=0, **kw):
    """fmt: "int8", "e4m3" or "" (a cache in dtype); new, old: (fewest, most) new tokens of a sequence and tokens before them."""
    return dict(op=op, dtype=dtype, fmt=fmt, B=B, new_lo=new[0], new_hi=new[1], old_lo=old[0], old_hi=old[1], H=H, H_kv=H_kv,
                D=D, P=P, window=window, packed=packed, rotary=rotary, adjacent=adjacent, most_kept=most_kept, **kw)


def listed():
    return [
        # one token of each of a batch: turned, quantised into its page, and read back
        _case("store", "bf16", "int8", 64, (1, 1), (1000, 30000), 32, 8, 128, rotary=128, name="store_tokens"),
        # pieces of prompts, the largest writes
        _case("store", "bf16", "e4m3", 4, (2001, 4500), (0, 5000), 32, 8, 128, rotary=128, name="store_prompts"),
        # a short sequence of a small fp32 layer is handed on in full precision
        _case("read", "f32", "e4m3", 1, (0, 0), (777, 777), 8, 2, 64, name="read_fp32"),
        # whole conversations are read back for a layer that selects tokens
        _case("read", "bf16", "int8", 4, (0, 0), (15001, 40000), 32, 8, 128, name="read_sequences"),
        # the smallest layer: one fp32 token over a short sequence
        _case("attn", "f32", "int8", 1, (1, 1), (4095, 4095), 8, 2, 64, packed=False, name="quant_token_fp32"),
        # a server's batch: one token of each of eight conversations of very different lengths
        _case("attn", "bf16", "int8", 8, (1, 1), (16384, 65536), 32, 8, 128, packed=False, name="quant_tokens_batch"),
        # a chunk of a long prompt over what its earlier chunks left
        _case("attn", "bf16", "e4m3", 1, (512, 512), (65536, 65536), 28, 4, 128, packed=False, name="quant_chunk_64k"),
        # a small tree of one short conversation
        _case("tree", "f32", "", 1, (13, 13), (1000, 1000), 8, 2, 64, packed=False, name="tree_small_fp32"),
        # trees of a batch of conversations
        _case("tree", "bf16", "", 16, (33, 64), (1000, 30000), 32, 8, 128, name="tree_batch"),
        # small trees over an 8-bit cache, in a layer that sees the last 4096 tokens only
        _case("tree", "bf16", "int8", 24, (5, 26), (3, 20000), 28, 4, 128, window=4096, name="tree_quant_window"),
        # the accepted paths of a batch
        _case("keep", "bf16", "", 64, (64, 64), (100, 5000), 32, 8, 128, most_kept=9, packed=False, name="keep_batch"),
        # and of a large one whose cache has 8 bits
        _case("keep", "bf16", "e4m3", 250, (20, 60), (5, 3000), 32, 8, 128, most_kept=7, name="keep_quant"),
    ]


def _spread(rng, lo, hi):
    """A whole number, spread evenly over its logarithm."""
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def _draw_one(rng):
    op = rng.choice(["store", "store", "read", "attn", "attn", "attn", "tree", "tree", "tree", "keep"])
    dtype, fmt = rng.choice(["bf16", "bf16", "f32"]), rng.choice(["int8", "e4m3"])
    H_kv = rng.choice([1, 2, 4, 8, 8, 16])
    H, D, P = H_kv * rng.choice([1, 2, 3, 4, 4, 5, 7, 8]), rng.choice([64, 128, 128]), rng.choice([8, 16, 16, 32, 64])
    window, packed = rng.choice([0, 0, 0, 1024, 4096]), rng.random() < 0.5
    if op == "store":
        B, n = _spread(rng, 1, 256), _spread(rng, 1, 8192)
        return _case(op, dtype, fmt, B, (max(1, n // rng.choice([1, 3, 50])), n), (rng.choice([0, 7]), _spread(rng, 8, 20000)),
                     H, H_kv, D, P, rotary=rng.choice([0, D, D, D // 2, 24]), adjacent=rng.choice([False, True]))
    if op == "read":
        n = _spread(rng, 1, 131072)
        return _case(op, dtype, fmt, _spread(rng, 1, 32), (0, 0), (max(1, n // rng.choice([1, 2, 5])), n), H, H_kv, D, P)
    if op == "attn":
        n, old = rng.choice([1, 1, _spread(rng, 2, 8), _spread(rng, 9, 4096)]), _spread(rng, 1, 131072)
        return _case(op, dtype, fmt, _spread(rng, 1, 32), (n if rng.random() < 0.5 else 1, n), (rng.choice([0, old // 4, old]), old),
                     H, H_kv, D, P, window, packed)
    fmt = rng.choice(["", "", fmt])
    n, old = _spread(rng, 2, 200), _spread(rng, 1, 65536)
    if op == "tree":
        return _case(op, dtype, fmt, _spread(rng, 1, 32), (n if rng.random() < 0.5 else 1, n), (rng.choice([0, old // 4, old]), old),
                     H, H_kv, D, P, window, packed)
    return _case(op, dtype, fmt, _spread(rng, 1, 256), (n, n), (0, min(old, 4000)), H, H_kv, D, P, most_kept=rng.randint(1, max(1, n // 2)))


def draw(rng):
    top = max(work(c)["flops"] for c in listed())
    while True:
        c = _draw_one(rng)
        if c["H"] > 128 or _tokens(c) * c["H_kv"] * c["D"] > 1 << 30:
            continue
        if not c["packed"]:
            c["new_lo"] = c["new_hi"]       # [B][C][H][D]: every sequence has as many
        w = work(c)
        if w["flops"] > top or w["bytes"] > 2e9 or w["bytes"] < 5e4:
            continue
        if c["op"] in ("attn", "tree"):
            scores = c["B"] * c["H"] * c["new_hi"] * (c["new_hi"] + c["old_hi"])
            if scores > 28 * 512 * 66048 or (c["dtype"] == "f32" and w["flops"] > top / 16):
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


def _cached(c):
    """Bytes of a token's K (or V) in the cache."""
    return c["H_kv"] * (c["D"] + 4 if c["fmt"] else c["D"] * _BYTES[c["dtype"]])


def _kept(c):
    """Accepted nodes of every sequence."""
    rng = random.Random("kept %(B)d %(most_kept)d" % c)
    return [rng.randint(0, min(c["most_kept"], n // 2)) for n in _lengths(c)[0]]


def work(case):
    c, es = case, _BYTES[case["dtype"]]
    row, q_row = c["H_kv"] * c["D"] * es, c["H"] * c["D"] * es
    new, old = _lengths(c)
    T = sum(new)
    if c["op"] == "store":      # rows in, codes out; codes in, rows out
        return dict(bytes=T * (2 * q_row + 4 * row + 4 * _cached(c)),
                    flops=T * (3.0 * (c["H"] + c["H_kv"]) * c["rotary"] + 8.0 * c["H_kv"] * c["D"]))
    if c["op"] == "read":
        return dict(bytes=2 * sum(old) * (row + _cached(c)), flops=2.0 * sum(old) * c["H_kv"] * c["D"])
    if c["op"] == "keep":
        return dict(bytes=4 * sum(_kept(c)) * _cached(c), flops=0)
    pairs, cached = 0, 0
    for n, o in zip(new, old):
        if c["op"] == "tree":   # every row sees itself and what is cached
            pairs += n * (min(o, c["window"] - 1) if c["window"] else o) + n
            cached += n + (min(o, c["window"] - 1) if c["window"] else o)
            continue
        w = c["window"] if c["window"] else n + o
        first = min(n, max(0, w - o))       # rows that the window does not cut
        pairs += first * o + first * (first + 1) // 2 + (n - first) * w
        cached += min(n + o, w + n - 1)
    return dict(bytes=2 * cached * _cached(c) + 2 * T * q_row + 4 * T * c["H"], flops=4.0 * pairs * c["H"] * c["D"])


# ---------------------------------------------------------------------------------------------------------------------
# inputs

def _gen(seed, salt=0):
    return torch.Generator(device=_DEV).manual_seed(int(seed) * 7919 + salt)


def _int32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device=_DEV)


def _encode(rows, fmt):
    """(codes, scales) of rows [..., D]; codes as int8 or e4m3.  In 64 bits: a quotient may lie next to the middle of two codes."""
    x = rows.double()
    m = x.abs().amax(dim=-1, keepdim=True)
    y = torch.where(m > 0, x * _TOP[fmt] / m, torch.zeros_like(x))
    if fmt == "int8":
        return y.round().to(torch.int8), (m / _TOP[fmt])[..., 0].float()
    behind = 4 - torch.frexp(y).exponent.clamp(min=-5)          # three bits behind the leading one, 2^-9 the smallest
    return torch.ldexp(torch.ldexp(y, behind).round(), -behind).to(torch.float8_e4m3fn), (m / _TOP[fmt])[..., 0].float()


def _pool(c, slots, g, x, name):
    """A pool of random rows [slots][heads][D], in pieces of 2^25 elements; scales [pages][heads][P]."""
    P, shape, step = c["P"], (slots, c["H_kv"], c["D"]), max(1, (1 << 25) // (c["P"] * c["H_kv"] * c["D"])) * c["P"]
    tdt = _TORCH[c["dtype"]]
    pool = torch.empty(shape, dtype=tdt if not c["fmt"] else torch.int8 if c["fmt"] == "int8" else torch.float8_e4m3fn, device=_DEV)
    scale = torch.empty((slots // P, c["H_kv"], P), device=_DEV) if c["fmt"] else None
    lean = x.get("lean_at") if name == "k" else None
    for a in range(0, slots, step):
        rows = torch.randn((min(step, slots - a),) + shape[1:], generator=g, device=_DEV)
        if lean is not None:
            mine = lean[(lean >= a) & (lean < a + step)] - a
            rows[mine] += x["lean"]
        rows = rows.to(tdt)
        if c["fmt"]:
            pool[a:a + step], mine = _encode(rows, c["fmt"])
            scale[a // P:(a + step) // P] = mine.view(-1, P, c["H_kv"]).transpose(1, 2)
        else:
            pool[a:a + step] = rows
    x[name + "_pool"], x[name + "_scale"] = pool, scale


def _inputs(c, seed):
    """What every pass of a case starts from; nothing in it depends on how the pass is computed."""
    g, P, D, H, H_kv, tdt, x = _gen(seed), c["P"], c["D"], c["H"], c["H_kv"], _TORCH[c["dtype"]], {}
    rng = random.Random("%d %d" % (seed, c["B"]))
    new, old = _lengths(c)
    if c["op"] == "read":
        new, old = old, new                 # every token of a sequence is asked for
    T, lens = sum(new), [n + o for n, o in zip(new, old)]
    need = [(n + P - 1) // P for n in lens]
    perm = torch.randperm(sum(need) + 3, generator=g, device=_DEV).int()
    x["indptr"], x["pages"] = _int32(np.cumsum([0] + need)), perm[:sum(need)].contiguous()
    x["lens"], x["max_len"] = _int32(lens), max(lens)
    x["q_indptr"], x["new"], x["rows"] = _int32(np.cumsum([0] + new)), max(new), T
    if c["op"] in ("attn", "tree"):
        # queries lean towards a direction that the first tokens' keys share: the logits of those stand out
        lean = torch.randn((H_kv, D), generator=g, device=_DEV)
        x["lean"] = 8.0 * lean / lean.norm(dim=-1, keepdim=True)
        x["q"] = (torch.randn((T, H, D), generator=g, device=_DEV) + x["lean"].repeat_interleave(H // H_kv, dim=0)).to(tdt)
        first = [(int(a) * P + np.arange(min(4, n))) for a, n in zip(np.cumsum([0] + need)[:-1], lens)]
        t = torch.tensor(np.concatenate(first), device=_DEV)
        x["lean_at"] = x["pages"][t // P].long() * P + t % P
    for name in "kv":
        _pool(c, perm.numel() * P, g, x, name)
    if c["op"] == "store":
        # one projection's output: q, k and v of a token follow each other
        qkv = torch.randn((T, (H + 2 * H_kv) * D), generator=g, device=_DEV).to(tdt)
        x["q"], x["k"], x["v"] = qkv[:, :H * D], qkv[:, H * D:(H + H_kv) * D], qkv[:, (H + H_kv) * D:]
        half = c["rotary"] // 2
        x["inv_freq"] = (1e6 ** -(torch.arange(half, device=_DEV, dtype=torch.float64) / max(1, half))).float()
    if c["op"] == "tree":                   # a node's parent is one of the nodes before it, a near one mostly
        x["parents"] = _int32([rng.randint(max(-1 if i == 0 else 0, i - 9), i - 1) if i > 0 else -1 for n in new for i in range(n)])
    if c["op"] == "keep":
        # accepted nodes: a few where they are, the others from behind (a pass leaves what the next one reads)
        kept, x["stride"] = _kept(c), max(1, c["most_kept"])
        x["path"] = torch.zeros((c["B"], x["stride"]), dtype=torch.int32, device=_DEV)
        for b, (m, n) in enumerate(zip(kept, new)):
            stay = rng.randint(0, m)
            nodes = list(range(stay)) + sorted(rng.sample(range(m, n), m - stay))
            if m:
                x["path"][b, :m] = _int32(nodes)
        x["count"], x["to_lens"] = _int32(kept), torch.zeros((c["B"],), dtype=torch.int32, device=_DEV)
    return x


def prepare(case, seed):
    c = case
    x = _inputs(c, seed)
    s = dict(c=c, x=x, sm=1.0 / math.sqrt(c["D"]))
    tdt, T, words = _TORCH[c["dtype"]], x["rows"], (x["new"] + 31) // 32
    empty = lambda shape, dtype=tdt: torch.zeros(shape, dtype=dtype, device=_DEV)
    if c["op"] in ("attn", "tree"):
        s["out"], s["lse"] = empty((T, c["H"], c["D"])), empty((T, c["H"]), torch.float32)
    if c["op"] == "tree":
        s["mask"], s["place"] = empty((T, words), torch.int32), empty((T,), torch.int32)
    if c["op"] == "store":
        s["q_out"] = empty((T, c["H"], c["D"]))
    if c["op"] in ("store", "read"):
        s["k_rows"], s["v_rows"] = empty((T, c["H_kv"], c["D"])), empty((T, c["H_kv"], c["D"]))
    if own:     # the handles of the layer's cache, the rotation and the workspace, which a program keeps
        from paper_2411_02886_amd import binding as ts
        s["ts"] = ts
        shape = (-1, c["P"], c["H_kv"], c["D"])
        pools = [None if c["fmt"] else x[n].view(shape) for n in ("k_pool", "v_pool")]
        s["problem"] = ts.Problem(batch=c["B"], chunk=x["new"], num_q_heads=c["H"], num_kv_heads=c["H_kv"], head_dim=c["D"],
                                  page_size=c["P"], max_seq_len=x["max_len"], dtype=ts.TS_BF16 if c["dtype"] == "bf16" else ts.TS_F32,
                                  k_pool=pools[0], v_pool=pools[1], page_indptr=x["indptr"], page_indices=x["pages"], seq_lens=x["lens"])
        s["quant"] = None
        if c["fmt"]:
            s["quant"] = ts.QuantCache(k_codes=x["k_pool"].view(shape), v_codes=x["v_pool"].view(shape), k_scale=x["k_scale"],
                                       v_scale=x["v_scale"], format=ts.TS_INT8 if c["fmt"] == "int8" else ts.TS_E4M3)
        s["ind"] = x["q_indptr"] if c["packed"] else None
        if c["op"] in ("attn", "tree"):
            n = (ts.ts_quant_attn_workspace_bytes if c["fmt"] else ts.ts_paged_attn_workspace_bytes)(s["problem"], T)
            s["ws"] = torch.empty(((n + 255) // 256 * 64,), dtype=torch.int32, device=_DEV)
        if c["op"] == "store":
            s["rope"] = ts.Rope(inv_freq=x["inv_freq"], adjacent=c["adjacent"]) if c["rotary"] else None
    return s


# ---------------------------------------------------------------------------------------------------------------------
# one pass

def _run_own(s):
    c, x, ts = s["c"], s["x"], s["ts"]
    p, quant, T, ind = s["problem"], s["quant"], x["rows"], s["ind"]
    if c["op"] in ("store", "read"):
        if c["op"] == "store":
            ts.ts_quant_append(p, quant, s["rope"], x["q"], x["k"], x["v"], x["q_indptr"], T, None, s["q_out"])
        ts.ts_quant_read(p, quant, x["q_indptr"], T, s["k_rows"], s["v_rows"])
        got = dict(k=s["k_rows"], v=s["v_rows"])
        return dict(got, q=s["q_out"], k_scale=x["k_scale"], v_scale=x["v_scale"]) if c["op"] == "store" else got
    if c["op"] == "keep":
        ts.ts_tree_keep(p, quant, x["path"], x["stride"], x["count"], ind, x["to_lens"])
        return _kept_pools(c, x)
    if c["op"] == "tree":
        ts.ts_tree_mask(p, x["parents"], ind, T, s["mask"], s["place"])
    mask = s["mask"] if c["op"] == "tree" else None
    if quant is not None:
        ts.ts_quant_attn(p, quant, x["q"], ind, T, c["window"], mask, s["sm"], s["out"], s["lse"], s["ws"])
    else:
        ts.ts_tree_attn(p, x["q"], ind, T, c["window"], mask, s["sm"], s["out"], s["lse"], s["ws"])
    got = dict(out=s["out"], lse=s["lse"])
    return dict(got, mask=s["mask"], place=s["place"]) if c["op"] == "tree" else got


def _kept_pools(c, x):
    """Moved rows are whole numbers or stored values: they have to be the same."""
    pools = {n: x[n].view(torch.int8) if c["fmt"] else x[n] for n in ("k_pool", "v_pool")}
    if c["fmt"]:
        pools.update(k_scale=x["k_scale"], v_scale=x["v_scale"])
    return dict(pools, lens=x["to_lens"])


def _row_places(x, P):
    """(sequence, place in it, pool row) of every new token: [T]."""
    row = torch.arange(x["rows"], device=_DEV)
    end = x["q_indptr"][1:].long()
    b = torch.bucketize(row, end, right=True)
    t = x["lens"].long()[b] - end[b] + row
    return b, t, x["pages"][x["indptr"][b].long() + t // P].long() * P + t % P


def _values(c, x, name, at):
    """Rows `at` of a pool as the values that they stand for, in 32 bits."""
    rows = x[name + "_pool"][at].float()
    return rows * x[name + "_scale"][at // c["P"], :, at % c["P"]][..., None] if c["fmt"] else rows


def _encode_rows(c, x, name, slot, rows):
    x[name + "_pool"][slot], x[name + "_scale"][slot // c["P"], :, slot % c["P"]] = _encode(rows, c["fmt"])


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


def _plain_store(s):
    c, x = s["c"], s["x"]
    T, tdt = x["rows"], _TORCH[c["dtype"]]
    b, t, slot = _row_places(x, c["P"])
    if c["op"] == "store":
        # in 64 bits: far places leave 32 no fraction of the angle, and a key's last bit may decide its code
        angle = t[:, None].double() * x["inv_freq"].double()
        cos, sin = angle.cos(), angle.sin()
        q = _turn(c, x["q"].view(T, c["H"], c["D"]).double(), cos, sin).to(tdt)
        k = _turn(c, x["k"].view(T, c["H_kv"], c["D"]).double(), cos, sin).to(tdt)
        _encode_rows(c, x, "k", slot, k)
        _encode_rows(c, x, "v", slot, x["v"].view(T, c["H_kv"], c["D"]))
    got = dict(k=_values(c, x, "k", slot).to(tdt), v=_values(c, x, "v", slot).to(tdt))
    return dict(got, q=q, k_scale=x["k_scale"], v_scale=x["v_scale"]) if c["op"] == "store" else got


def _plain_keep(s):
    c, x = s["c"], s["x"]
    count, path = x["count"].long()[:, None], x["path"].long()
    n = (x["q_indptr"][1:] - x["q_indptr"][:-1]).long()[:, None]
    base = x["lens"].long()[:, None] - n
    i = torch.arange(x["stride"], device=_DEV)[None, :].expand_as(path)
    at = lambda t: x["pages"][(x["indptr"][:-1, None].long() + t // c["P"])[i < count]].long() * c["P"] + (t % c["P"])[i < count]
    src, dst = at(base + path), at(base + i)
    for name in "kv":
        pool, scale = x[name + "_pool"], x[name + "_scale"]
        if c["fmt"]:
            pool = pool.view(torch.int8)
            scale[dst // c["P"], :, dst % c["P"]] = scale[src // c["P"], :, src % c["P"]]
        pool[dst] = pool[src]
    x["to_lens"].copy_((base + count)[:, 0])
    return _kept_pools(c, x)


def _plain_mask(s):
    """Which new tokens see which, [B][C][C], from the parents: the closure of "is the parent of"; places; the bits as words."""
    c, x = s["c"], s["x"]
    B, C, T = c["B"], x["new"], x["rows"]
    b, t, _ = _row_places(x, c["P"])
    i = torch.arange(T, device=_DEV) - x["q_indptr"][:-1].long()[b]
    par = x["parents"].long()
    see = torch.zeros((B, C, C), device=_DEV)
    see[b, i, i] = 1.0
    see[b, i, par.clamp(min=0)] = torch.maximum(see[b, i, par.clamp(min=0)], (par >= 0).float())
    for _ in range(max(1, C.bit_length())):
        see = (torch.bmm(see, see) > 0).float()
    see = see > 0
    rows = see[b, i]                                                                    # [T][C]
    words = (C + 31) // 32
    bits = torch.zeros((T, words * 32), dtype=torch.int64, device=_DEV)
    bits[:, :C] = rows
    word = (bits.view(T, words, 32) << torch.arange(32, device=_DEV)).sum(dim=-1)
    word = torch.where(word >= 1 << 31, word - (1 << 32), word).int()
    return see, word, (t - i + rows.sum(dim=-1) - 1).int()


def _plain_attn(s):
    c, x = s["c"], s["x"]
    B, H, H_kv, D, P, T = c["B"], c["H"], c["H_kv"], c["D"], c["P"], x["rows"]
    G, C, N = H // H_kv, x["new"], x["max_len"]
    start = x["q_indptr"][:-1].long()
    new = x["q_indptr"][1:].long() - start
    base = x["lens"].long() - new
    chunk, t = torch.arange(C, device=_DEV), torch.arange(N, device=_DEV)
    q = x["q"][(start[:, None] + chunk).clamp(max=T - 1)].float()                       # [B][C][H][D]
    q = q.view(B, C, H_kv, G, D).permute(0, 2, 1, 3, 4).reshape(B * H_kv, C * G, D)
    at = x["indptr"][:-1, None].long() + (t // P)[None, :]
    slot = x["pages"][at.clamp(max=x["pages"].numel() - 1)].long() * P + t % P
    k = _values(c, x, "k", slot).permute(0, 2, 3, 1).reshape(B * H_kv, D, N)
    got = {}
    if c["op"] == "tree":
        see, got["mask"], got["place"] = _plain_mask(s)
        j = t[None, :] - base[:, None]                                                  # [B][N] which new token
        seen = see.gather(2, j.clamp(min=0, max=C - 1)[:, None, :].expand(B, C, N)) & (j < new[:, None])[:, None, :]
        cached = (j < 0)[:, None, :]
        if c["window"]:
            cached = cached & (t[None, None, :] >= (base[:, None] + see.sum(dim=-1) - c["window"])[:, :, None])
        seen = torch.where((j < 0)[:, None, :], cached, seen)
    else:
        pos = base[:, None] + chunk                                                     # [B][C]
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
    v = _values(c, x, "v", slot).permute(0, 2, 1, 3).reshape(B * H_kv, N, D)
    o = torch.bmm(weights.view(B * H_kv, C * G, N), v).view(B, H_kv, C, G, D) / total.clamp(min=1e-38)
    lse = (top + total.log())[..., 0]
    row = torch.arange(T, device=_DEV)
    b = torch.bucketize(row, x["q_indptr"][1:].long(), right=True)
    o = o.permute(0, 2, 1, 3, 4).reshape(B, C, H, D)[b, row - start[b]]
    lse = lse.permute(0, 2, 1, 3).reshape(B, C, H)[b, row - start[b]]
    return dict(got, out=o.to(s["out"].dtype), lse=lse)


def run(state):
    if own:
        return _run_own(state)
    return {"store": _plain_store, "read": _plain_store, "keep": _plain_keep, "attn": _plain_attn, "tree": _plain_attn}[state["c"]["op"]](state)


# ---------------------------------------------------------------------------------------------------------------------
# the same in 64 bits, sequence by sequence

def _exact_rows(c, rows):
    """(values after quantising, scales) of rows [..., D] of stored numbers, in 64 bits."""
    rows, top = rows.double(), _TOP[c["fmt"]]
    m = rows.abs().max(dim=-1).values
    z = rows * top / torch.where(m > 0, m, torch.ones_like(m))[..., None]       # (a tie comes out as one)
    if c["fmt"] == "int8":
        code = z.round()
    else:                                   # three bits behind the leading one, steps of 2^-9 at least; a tie goes to the even one
        step = torch.exp2(torch.floor(torch.log2(z.abs().clamp(min=2.0 ** -6))) - 3)
        code = (z / step).round() * step
    return code * (m / top)[..., None], m / top


def _exact_store(c, x):
    H, H_kv, D, P, tdt = c["H"], c["H_kv"], c["D"], c["P"], _TORCH[c["dtype"]]
    new, old = _lengths(c)
    if c["op"] == "read":
        new, old = old, new
    place = torch.cat([torch.arange(o, o + n, device=_DEV) for n, o in zip(new, old)])
    page = torch.cat([x["pages"].long()[int(a) + torch.arange(o, o + n, device=_DEV) // P]
                      for a, n, o in zip(x["indptr"].tolist(), new, old)])
    slot = page * P + place % P
    if c["op"] == "read":
        return {n: x[n + "_pool"][slot].double() * x[n + "_scale"].transpose(1, 2).reshape(-1, H_kv)[slot].double()[..., None] for n in "kv"}
    q, k, v = (x[n].double().view(-1, h, D).clone() for n, h in (("q", H), ("k", H_kv), ("v", H_kv)))
    for i in range(c["rotary"] // 2):
        z = torch.polar(torch.ones_like(place, dtype=torch.float64), place.double() * float(x["inv_freq"][i]))[:, None]
        e0, e1 = (2 * i, 2 * i + 1) if c["adjacent"] else (i, i + c["rotary"] // 2)
        for rows in (q, k):
            w = torch.complex(rows[..., e0], rows[..., e1]) * z
            rows[..., e0], rows[..., e1] = w.real, w.imag
    got = dict(q=q)
    for n, rows in (("k", k.to(tdt)), ("v", v)):        # what a cache of the layer's type would hold is quantised
        got[n], scale = _exact_rows(c, rows)
        flat = x[n + "_scale"].double().transpose(1, 2).reshape(-1, H_kv)
        flat[slot] = scale
        got[n + "_scale"] = flat.view(-1, P, H_kv).transpose(1, 2)
    return got


def _exact_keep(c, x):
    P, (new, old) = c["P"], _lengths(c)
    pools = _kept_pools(c, x)
    of = torch.arange(x["k_pool"].shape[0], device=_DEV)
    for b, m in enumerate(_kept(c)):
        place = lambda t: x["pages"].long()[int(x["indptr"][b]) + t // P] * P + t % P
        of[place(old[b] + torch.arange(m, device=_DEV))] = place(old[b] + x["path"][b, :m].long())
    got = {}
    for n in pools:
        if n.endswith("pool"):
            got[n] = pools[n][of] if c["fmt"] else pools[n][of].double()
        elif n.endswith("scale"):
            flat = pools[n].transpose(1, 2).reshape(-1, c["H_kv"])[of]
            got[n] = flat.view(-1, P, c["H_kv"]).transpose(1, 2).double()
    return dict(got, lens=_int32([o + m for o, m in zip(old, _kept(c))]))


def _exact_attn(c, x):
    T, H, D, P, H_kv = x["rows"], c["H"], c["D"], c["P"], c["H_kv"]
    G = H // H_kv
    out = torch.zeros((T, H, D), dtype=torch.float64, device=_DEV)
    lse = torch.full((T, H), -math.inf, dtype=torch.float64, device=_DEV)
    new, old = _lengths(c)
    words, word, place = (x["new"] + 31) // 32, [], []
    pages, first, row = x["pages"].long(), x["indptr"].tolist(), 0
    for b, (n, o) in enumerate(zip(new, old)):
        N = n + o
        t = torch.arange(N, device=_DEV)
        slot = pages[first[b] + t // P] * P + t % P
        hidden = t[None, :] > o + torch.arange(n, device=_DEV)[:, None]
        at = o + torch.arange(n, device=_DEV)
        if c["op"] == "tree":
            path = []                       # of each node the nodes from the root to it
            for i, parent in enumerate(x["parents"][row:row + n].tolist()):
                path.append((path[parent] if parent >= 0 else []) + [i])
            sees = np.zeros((n, n), dtype=bool)
            for i, nodes in enumerate(path):
                sees[i, nodes] = True
                word.append([sum(1 << (j - 32 * w) for j in nodes if j // 32 == w) for w in range(words)])
                place.append(o + len(nodes) - 1)
            hidden[:, o:] = torch.tensor(~sees, device=_DEV)
            at = torch.tensor(place[row:], device=_DEV)
        if c["window"]:
            far = t[None, :] <= at[:, None] - c["window"]
            if c["op"] == "tree":
                far[:, o:] = False
            hidden = hidden | far
        step = max(1, (1 << 28) // max(1, N * G))
        for kv in range(H_kv):
            k, v = (x[p + "_pool"][slot, kv].double() for p in "kv")
            if c["fmt"]:
                k, v = (r * x[p + "_scale"][slot // P, kv, slot % P].double()[:, None] for p, r in (("k", k), ("v", v)))
            for a in range(0, n, step):
                m = min(step, n - a)
                qs = x["q"][row + a:row + a + m, kv * G:(kv + 1) * G].double().reshape(m * G, D)
                z = (qs @ k.t().contiguous() / math.sqrt(D)).view(m, G, N)
                z.masked_fill_(hidden[a:a + m, None, :], -math.inf)
                l = torch.logsumexp(z, dim=-1)
                out[row + a:row + a + m, kv * G:(kv + 1) * G] = (torch.exp(z - l[..., None]).view(m * G, N) @ v).view(m, G, D)
                lse[row + a:row + a + m, kv * G:(kv + 1) * G] = l
        row += n
    if c["op"] == "tree":
        return dict(out=out, lse=lse, place=_int32(place),
                    mask=torch.tensor(np.array(word, dtype=np.uint32).view(np.int32), device=_DEV))
    return dict(out=out, lse=lse)


def exact(case, seed):
    x = _inputs(case, seed)
    return {"store": _exact_store, "read": _exact_store, "keep": _exact_keep, "attn": _exact_attn, "tree": _exact_attn}[case["op"]](case, x)
