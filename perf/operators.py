"""Operators around the decode step, timed: their plain forms in elementary torch operations, the calls that a program
makes of the library, what a pass cannot do without, and the same results in 64 bits.

  append   rotary positions of new tokens' queries and keys, and the new rows into a bf16 cache (rk_rope_append)
  append8  the same into a cache of 8 bits, whose blocks are quantised as they fill (rk_rope_append_q8)
  attn8    one decode step over a cache of 8 bits, with its weights or without (rk_full_attn_q8)
  gather8  selected rows of a cache of 8 bits into the bf16 small cache (rk_gather_small_kv_q8)
  prompt   attention of several new tokens of each sequence, whole prompts, chunks or one token, with capped scores, a bias
           by distance, document and prefix masks (rk_prompt_attn)

Heads, lengths and batches are those of the benchmark's workloads (32 heads over 8 and 28 over 4, 2k to 128k rows, a ragged
batch of 16), odd ones between them.  A cache of 8 bits keeps whole blocks of tokens as e4m3 or int8 with one power of two per block
and KV head as its scale, and the rows of the block that is not full yet in bf16.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))
FORMATS = {"e4m3": (torch.float8_e4m3fn, 448.0), "int8": (torch.int8, 127.0)}


def _case(name, kind, **changes):
    c = {"kind": kind, "batch": 1, "hq": 32, "hkv": 8, "len": 2048, "min_len": 0, "shape": 1}
    c.update(changes)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: one new token of one sequence on its way into the cache; latency decides
        _case("append_step", "append", new=1, len=2001, rot=128, interleaved=False),
        # a prompt of a model that rotates half of the head, pairs side by side: bound by memory
        _case("append_prompt_8k", "append", new=8192, len=8192, rot=64, interleaved=True),
        # one token of each sequence of a served batch into e4m3, some of them filling a block
        _case("append8_batch64", "append8", batch=64, hq=28, hkv=4, new=1, len=1024, min_len=200, rot=128, interleaved=False,
              fmt="e4m3", block=32),
        # ragged prompts into int8
        _case("append8_prompts", "append8", batch=5, new=2048, len=2048, min_len=300, rot=128, interleaved=False, fmt="int8",
              block=64),
        # a decode step at 32k rows that returns its weights for the selection, at an odd length
        _case("attn8_32k", "attn8", len=32777, fmt="e4m3", block=32, weights=True),
        # a served batch with ragged lengths, no weights, 7 query heads to a KV head, int8
        _case("attn8_ragged16", "attn8", batch=16, hq=28, hkv=4, len=16384, min_len=4096, fmt="int8", block=64, weights=False),
        # the longest context, with the weights
        _case("attn8_128k", "attn8", len=131072, fmt="e4m3", block=128, weights=True),
        # the small cache of a refresh out of a cache of 8 bits
        _case("gather8_2k", "gather8", len=32777, fmt="e4m3", block=32, k=2048),
        # ... of a ragged batch
        _case("gather8_batch16", "gather8", batch=16, len=16384, min_len=4096, fmt="int8", block=64, k=1024),
        # a whole prompt, causal: the largest, bound by the matrix instructions
        _case("prompt_8k", "prompt", new=8192, len=8192, cap=0.0, slopes=False, docs=0, prefix=0),
        # chunks of prompts behind what is cached already, packed documents with a prefix that sees itself both ways, capped scores
        _case("prompt_chunks", "prompt", batch=3, hq=28, hkv=4, new=700, len=9001, min_len=900, cap=30.0, slopes=False, docs=3, prefix=40),
        # one token of each sequence, with a bias by distance
        _case("prompt_step", "prompt", batch=8, new=1, len=16384, min_len=2048, cap=0.0, slopes=True, docs=0, prefix=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append8", "append8", "attn8", "attn8", "gather8", "prompt", "prompt", "prompt"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (28, 4), (8, 8), (16, 8), (64, 8), (20, 4), (5, 1)])
    c = _case(None, kind, hq=hq, hkv=hkv, shape=rng.randint(1, 10 ** 6))
    if kind in ("append", "append8"):
        c["new"] = rng.choice([1, _log_int(rng, 2, 8192)])
        c["batch"] = max(1, min(_log_int(rng, 1, 64), 8192 // c["new"]))
        c["rot"], c["interleaved"] = rng.choice([128, 128, 64, 32, 96]), rng.random() < 0.4
        c["len"] = c["new"] if c["new"] > 1 else _log_int(rng, 130, 4096)
    else:
        c["batch"] = rng.choice([1, 1, _log_int(rng, 2, 16)])
        c["len"] = min(_log_int(rng, 500, 131072), 131072 * 8 // (c["batch"] * hkv))
    if kind in ("append8", "attn8", "gather8"):
        c["fmt"], c["block"] = rng.choice(["e4m3", "int8"]), rng.choice([16, 32, 64, 128])
    if kind == "attn8":
        c["weights"] = rng.random() < 0.5
    if kind == "gather8":
        c["k"] = max(16, min(8192, c["len"] // rng.randint(8, 16)))
    if kind == "prompt":
        c["len"] = min(c["len"], 32768)
        c["new"] = rng.choice([1, 1, _log_int(rng, 2, 8192), _log_int(rng, 2, 8192)])
        most = 8192 * 8192 * 32 // 2                     # (query head, row) pairs of the largest case
        c["new"] = max(1, min(c["new"], c["len"], most // (c["batch"] * hq * c["len"])))
        c["cap"], c["slopes"] = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.random() < 0.4
        c["docs"], c["prefix"] = rng.choice([0, 0, 1, 4]), rng.choice([0, 0, 64, 500])
    if c["batch"] > 1 and rng.random() < 0.7 and kind != "append":
        c["min_len"] = max(1, c["len"] // rng.randint(2, 6))
    return c


# ---- shapes, a function of the case alone -------------------------------------------------------

def _lens(c):
    """Rows of every sequence, the new tokens included (host numbers)."""
    n = int(c["len"])
    if not c["min_len"]:
        return [n] * c["batch"]
    r = random.Random(c["shape"])
    return [n] + [r.randint(c["min_len"], n) for _ in range(c["batch"] - 1)]


def _new_lens(c):
    return [min(int(c["new"]), n) for n in _lens(c)]


def _ranges(c):
    """first, end: the rows that each new token sees, int32 [batch, new] on the host; (None, None) for the plain causal mask.
    docs: documents packed one behind the other start at so many random rows more; prefix: the first rows of each document
    are seen by all of it."""
    if not c["docs"] and not c["prefix"]:
        return None, None
    r = np.random.default_rng(c["shape"])
    first = np.zeros((c["batch"], c["new"]), np.int32)
    end = np.zeros((c["batch"], c["new"]), np.int32)
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        starts = np.unique(np.concatenate([[0], r.integers(0, n, c["docs"])]))
        p = np.arange(n - new, n)
        which = np.searchsorted(starts, p, side="right") - 1
        stops = np.append(starts[1:], n)
        first[b, :new] = starts[which]
        end[b, :new] = np.maximum(p + 1, np.minimum(starts[which] + c["prefix"], stops[which]))
    return first, end


def _pairs(c):
    """(new token, row) pairs that the masks leave."""
    first, end = _ranges(c)
    if first is not None:
        return int((end.astype(np.int64) - first).sum())
    return sum(new * (n - new) + new * (new + 1) // 2 for n, new in zip(_lens(c), _new_lens(c)))


# ---- inputs -------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _up(n, m):
    return (n + m - 1) // m * m


def _table(c):
    """cos and sin of every position, fp32 [positions, rot]: the angles in 64 bits."""
    half = c["rot"] // 2
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a = torch.arange(c["len"], dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _quantise(x, fmt):
    """Whole blocks [..., block, D] in fp32 -> (8 bits, scale): the smallest power of two that brings the largest
    value into the type's range."""
    dtype, most = FORMATS[fmt]
    top = x.abs().amax(dim=(-1, -2))
    m, e = torch.frexp(top / most)                       # top / most = m 2^e, 1/2 <= m < 1
    scale = torch.where(top > 0, torch.ldexp(torch.ones_like(top), (e - (m == 0.5).int()).clamp(min=-126)), torch.ones_like(top))
    y = x / scale[..., None, None]
    return (torch.round(y) if fmt == "int8" else y).to(dtype), scale


def _cache8(c, g, lens):
    """A cache of 8 bits that holds `lens` rows of random keys and values of varied size."""
    B, H, blk = c["batch"], c["hkv"], c["block"]
    rows = _up(max(lens), blk)
    s = {}
    for n in ("k", "v"):
        x = _normal(g, B, H, rows, D).float().view(B, H, rows // blk, blk, D)
        x = x * torch.exp(0.5 * torch.randn(B, H, rows // blk, 1, 1, generator=g, device="cuda"))
        x8, s[n + "_scale"] = _quantise(x.to(torch.bfloat16).float(), c["fmt"])
        s[n + "8"] = x8.view(B, H, rows, D)
        s[n + "_tail"] = _normal(g, B, H, blk, D)
    return s


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, Hq, H = c["batch"], c["hq"], c["hkv"]
    lens = _lens(c)
    s = {"c": c, "seq_lens": _int32(lens)}
    if c["kind"] in ("append", "append8"):
        T = c["new"]
        # the rows of one fused projection, as a layer has them
        qkv = _normal(g, B, T, Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        s["table"], s["new_lens"] = _table(c), _int32(_new_lens(c))
        s["q_out"] = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
        if c["kind"] == "append":
            rows = _up(max(lens), 64)
            s["K"], s["V"] = _normal(g, B, H, rows, D), _normal(g, B, H, rows, D)
        else:
            s.update(_cache8(c, g, lens))
    elif c["kind"] in ("attn8", "gather8"):
        s.update(_cache8(c, g, lens))
        if c["kind"] == "attn8":
            s["q"] = _normal(g, B, Hq, D)
            s["out"] = torch.zeros(B, Hq, D, dtype=torch.bfloat16, device="cuda")
            s["lse"] = torch.zeros(B, Hq, device="cuda")
            s["weights"] = torch.zeros(B, Hq, _up(c["len"], 64), device="cuda") if c["weights"] else None
        else:
            k = c["k"]
            idx = torch.full((B, H, k), -1, dtype=torch.int32, device="cuda")
            for b, n in enumerate(lens):                 # distinct rows in the order of their scores: any order
                kk = min(k, n)
                idx[b, :, :kk] = torch.rand(H, n, generator=g, device="cuda").argsort(dim=1)[:, :kk].int()
            s["idx"] = idx
            s["small_K"] = torch.zeros(B, H, k, D, dtype=torch.bfloat16, device="cuda")
            s["small_V"] = torch.zeros_like(s["small_K"])
            s["tail_start"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    else:
        rows = _up(max(lens), 64)
        gain = 4.0 if c["cap"] else 1.0                  # scores that the cap bends
        s["q"] = (_normal(g, B, c["new"], Hq, D).float() * gain).to(torch.bfloat16)
        s["K"], s["V"] = _normal(g, B, H, rows, D), _normal(g, B, H, rows, D)
        s["new_lens"] = _int32(_new_lens(c))
        first, end = _ranges(c)
        s["first"], s["end"] = (None, None) if first is None else (torch.from_numpy(first).cuda(), torch.from_numpy(end).cuda())
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, Hq + 1, device="cuda") / Hq) if c["slopes"] else None
        s["out"] = torch.zeros(B, c["new"], Hq, D, dtype=torch.bfloat16, device="cuda")
        s["lse"] = torch.zeros(B, c["new"], Hq, device="cuda")
    return s


# ---- one pass -----------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["c"]["kind"]](s)


def _plain_rotate(x, cos, sin, c):
    """x [B, T, heads, D] in fp32, cos and sin [B, T, 1, rot / 2]."""
    rot, half = c["rot"], c["rot"] // 2
    r, rest = x[..., :rot], x[..., rot:]
    if c["interleaved"]:
        a, b = r[..., 0::2], r[..., 1::2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = r[..., :half], r[..., half:]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([y, rest], dim=-1).to(torch.bfloat16)


def _plain_rotated(s):
    """The new rows of q, k and v, their rows in the cache [B, T] and which of them there are."""
    c, T = s["c"], s["c"]["new"]
    i = torch.arange(T, device="cuda")
    row = (s["seq_lens"] - s["new_lens"])[:, None] + i
    real = i < s["new_lens"][:, None]
    t = s["table"][row.clamp(0, c["len"] - 1).long()][:, :, None]
    cos, sin = t[..., :c["rot"] // 2], t[..., c["rot"] // 2:]
    q, k = (_plain_rotate(s[n].float(), cos, sin, c) for n in ("q", "k"))
    return q, k, s["v"], row.long(), real


def _plain_append(s):
    q, k, v, row, real = _plain_rotated(s)
    s["q_out"][real] = q[real]
    b = torch.arange(s["c"]["batch"], device="cuda")[:, None].expand_as(row)[real]
    s["K"][b, :, row[real]] = k[real]
    s["V"][b, :, row[real]] = v[real]
    return {"q": s["q_out"], "K": s["K"], "V": s["V"]}


def _plain_append8(s):
    c, blk, B = s["c"], s["c"]["block"], s["c"]["batch"]
    q, k, v, row, real = _plain_rotated(s)
    s["q_out"][real] = q[real]
    n, start = s["seq_lens"].long(), (s["seq_lens"] - s["new_lens"]).long()
    b = torch.arange(B, device="cuda")
    # the blocks that hold new rows, in bf16: rows that were there already come from the tail
    b0, nb = start // blk, (c["new"] + blk - 2) // blk + 1
    wide = torch.zeros(B, c["hkv"], nb * blk, D, dtype=torch.bfloat16, device="cuda")
    ids = b[:, None].expand_as(row)[real]
    number = b0[:, None] + torch.arange(nb, device="cuda")
    whole = ((number + 1) * blk <= n[:, None]) & (number * blk < n[:, None])
    last = (n - 1) // blk
    part = (n % blk != 0) & (s["new_lens"] > 0)
    slot = torch.arange(blk, device="cuda")
    for x, name in ((k, "k"), (v, "v")):                 # (keys, then values)
        w = wide.clone()
        w[:, :, :blk] = s[name + "_tail"]
        w[ids, :, (row - (b0 * blk)[:, None])[real]] = x[real]
        x8, scale = _quantise(w.view(B, c["hkv"], nb, blk, D).float(), c["fmt"])
        wb, wn = torch.nonzero(whole, as_tuple=True)
        at = number[wb, wn]
        s[name + "8"].view(torch.uint8).view(B, c["hkv"], -1, blk, D)[wb, :, at] = x8.view(torch.uint8)[wb, :, wn]
        s[name + "_scale"][wb, :, at] = scale[wb, :, wn]
        # the last block, where it is not full: its new rows go to the tail
        pos = (last * blk)[:, None] + slot
        new = part[:, None] & (pos >= start[:, None]) & (pos < n[:, None])
        tb, ts = torch.nonzero(new, as_tuple=True)
        s[name + "_tail"][tb, :, ts] = w[tb, :, (pos - (b0 * blk)[:, None])[tb, ts]]
    return {"q": s["q_out"], **{n: s[n] for n in ("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail")}}


def _plain_rows8(s, name):
    """The values that a cache of 8 bits stands for, fp32 [B, H, rows, D]."""
    blk, x8 = s["c"]["block"], s[name + "8"]
    B, H, rows, _ = x8.shape
    x = (x8.float().view(B, H, rows // blk, blk, D) * s[name + "_scale"][..., None, None]).view(B, H, rows, D)
    j = torch.arange(rows, device="cuda")
    in_tail = j >= (s["seq_lens"] // blk * blk)[:, None]
    return torch.where(in_tail[:, None, :, None], s[name + "_tail"].float()[:, :, j % blk], x)


def _plain_attn8(s):
    c, B, Hq, H = s["c"], s["c"]["batch"], s["c"]["hq"], s["c"]["hkv"]
    k, v = _plain_rows8(s, "k"), _plain_rows8(s, "v")
    rows = k.shape[2]
    sc = torch.matmul(s["q"].float().view(B, H, Hq // H, D), k.transpose(2, 3)) * SCALE
    sc = sc.masked_fill((torch.arange(rows, device="cuda") >= s["seq_lens"][:, None])[:, None, None], -math.inf)
    m = sc.amax(dim=-1, keepdim=True)
    p = torch.exp(sc - m)
    total = p.sum(dim=-1, keepdim=True)
    w = p / total
    s["out"].copy_(torch.matmul(w, v).view(B, Hq, D))
    s["lse"].copy_((m + torch.log(total)).view(B, Hq))
    if s["weights"] is None:
        return {"out": s["out"], "lse": s["lse"]}
    n = min(rows, s["weights"].shape[2])
    s["weights"][:, :, :n] = w.view(B, Hq, rows)[:, :, :n]
    return {"out": s["out"], "lse": s["lse"], "weights": s["weights"]}


def _plain_gather8(s):
    blk, idx = s["c"]["block"], s["idx"]
    B, H, k = idx.shape
    j = idx.clamp(min=0).long()
    in_tail = j >= (s["seq_lens"] // blk * blk)[:, None, None]
    b, h = torch.arange(B, device="cuda")[:, None, None], torch.arange(H, device="cuda")[:, None]
    for n, small in (("k", "small_K"), ("v", "small_V")):
        x = s[n + "8"].view(torch.uint8)[b, h, j].view(s[n + "8"].dtype).float() * s[n + "_scale"][b, h, j // blk][..., None]
        x = torch.where(in_tail[..., None], s[n + "_tail"][b, h, j % blk].float(), x).to(torch.bfloat16)
        s[small].copy_(torch.where((idx >= 0)[..., None], x, s[small]))
    s["tail_start"].copy_(s["seq_lens"])
    return {"small_K": s["small_K"], "small_V": s["small_V"], "tail_start": s["tail_start"]}


def _plain_prompt(s):
    c, B, Hq, H, T = s["c"], s["c"]["batch"], s["c"]["hq"], s["c"]["hkv"], s["c"]["new"]
    G, rows = Hq // H, s["K"].shape[2]
    p = (s["seq_lens"] - s["new_lens"])[:, None] + torch.arange(T, device="cuda")
    real = torch.arange(T, device="cuda") < s["new_lens"][:, None]
    j = torch.arange(rows, device="cuda")
    first = torch.zeros_like(p) if s["first"] is None else s["first"]
    end = p + 1 if s["end"] is None else s["end"]
    hidden = (j < first[..., None]) | (j >= end[..., None]) | (j >= s["seq_lens"][:, None, None])
    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * T, D)
    sc = torch.matmul(q, s["K"].float().transpose(2, 3)).view(B, H, G, T, rows) * SCALE
    if c["cap"]:
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    if s["slopes"] is not None:
        sc = sc - s["slopes"].view(H, G, 1, 1) * (p[..., None] - j).abs().float()[:, None, None]
    sc = sc.masked_fill(hidden[:, None, None], -math.inf)
    m = sc.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    w = torch.exp(sc - m)
    total = w.sum(dim=-1, keepdim=True)
    w = torch.where(total > 0, w / total, torch.zeros_like(w))
    out = torch.matmul(w.view(B, H, G * T, rows), s["V"].float()).view(B, H, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    lse = (m + torch.log(total)).view(B, Hq, T).permute(0, 2, 1)
    s["out"].copy_(torch.where(real[..., None, None], out.to(torch.bfloat16), s["out"]))
    s["lse"].copy_(torch.where(real[..., None], lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


_plain = {"append": _plain_append, "append8": _plain_append8, "attn8": _plain_attn8, "gather8": _plain_gather8, "prompt": _plain_prompt}


def _handles(s):
    """What a program makes once and keeps: geometry, the rotary table's handle, the cache, the scratch."""
    if "geom" not in s:
        import paper_2411_05787_amd as rk
        c = s["c"]
        s["rk"], s["geom"] = rk, rk.Geom(c["batch"], c["hq"], c["hkv"], D, SCALE)
        if "table" in s:
            s["rope"] = rk.Rope(s["table"], interleaved=c["interleaved"])
        if "k8" in s:
            s["cache"] = rk.Kv8(s["geom"], s["k8"], s["v8"], s["k_scale"], s["v_scale"], s["k_tail"], s["v_tail"])
        if c["kind"] == "attn8":
            s["ws"] = rk.Workspace(s["geom"], c["len"], 1)
        elif c["kind"] == "prompt":
            s["ws"] = rk.PromptWorkspace(s["geom"], c["new"], c["len"])
    return s["rk"], s["geom"]


def _own_append(s):
    rk, geom = _handles(s)
    rk.rk_rope_append(geom, s["q"], s["k"], s["v"], s["rope"], s["K"], s["V"], s["seq_lens"], s["q_out"], new_lens=s["new_lens"])
    return {"q": s["q_out"], "K": s["K"], "V": s["V"]}


def _own_append8(s):
    rk, geom = _handles(s)
    rk.rk_rope_append_q8(geom, s["q"], s["k"], s["v"], s["rope"], s["cache"], s["seq_lens"], s["q_out"], new_lens=s["new_lens"])
    return {"q": s["q_out"], **{n: s[n] for n in ("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail")}}


def _own_attn8(s):
    rk, geom = _handles(s)
    rk.rk_full_attn_q8(geom, s["q"], s["cache"], s["seq_lens"], s["c"]["len"], s["out"], weights=s["weights"], lse=s["lse"],
                       workspace=s["ws"])
    return {"out": s["out"], "lse": s["lse"], **({} if s["weights"] is None else {"weights": s["weights"]})}


def _own_gather8(s):
    rk, geom = _handles(s)
    rk.rk_gather_small_kv_q8(geom, s["cache"], s["idx"], s["c"]["k"], s["small_K"], s["small_V"], s["seq_lens"],
                             tail_start=s["tail_start"])
    return {"small_K": s["small_K"], "small_V": s["small_V"], "tail_start": s["tail_start"]}


def _own_prompt(s):
    rk, geom = _handles(s)
    rk.rk_prompt_attn(geom, s["q"], s["K"], s["V"], s["seq_lens"], s["c"]["len"], s["out"], new_lens=s["new_lens"],
                      first=s["first"], end=s["end"], cap=s["c"]["cap"], slopes=s["slopes"], lse=s["lse"], workspace=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


_own = {"append": _own_append, "append8": _own_append8, "attn8": _own_attn8, "gather8": _own_gather8, "prompt": _own_prompt}


# ---- what a pass cannot do without --------------------------------------------------------------

def work(c):
    lens, Hq, H = _lens(c), c["hq"], c["hkv"]
    if c["kind"] in ("append", "append8"):
        n = sum(_new_lens(c))
        rows = n * (2 * Hq + 2 * H) * D * 2 + n * c["rot"] * 4
        if c["kind"] == "append":
            return {"bytes": rows + n * 2 * H * D * 2, "flops": n * (Hq + H) * 3 * c["rot"]}
        blk, full, tail, old = c["block"], 0, 0, 0
        for m, new in zip(lens, _new_lens(c)):
            start = m - new
            full += m // blk - start // blk                                  # blocks that fill
            tail += min(m % blk, new)                                        # rows that stay in bf16
            old += start % blk if m // blk > start // blk else 0             # ... and come back from there
        return {"bytes": rows + 2 * H * (full * (blk * D + 4) + (tail + old) * D * 2), "flops": n * (Hq + H) * 3 * c["rot"]}
    if c["kind"] == "attn8":
        rows = sum(n // c["block"] * (c["block"] * D + 4) + n % c["block"] * D * 2 for n in lens)
        return {"bytes": 2 * H * rows + (4 * Hq * sum(lens) if c["weights"] else 0) + c["batch"] * Hq * (4 * D + 4),
                "flops": 4 * D * Hq * sum(lens)}
    if c["kind"] == "gather8":
        rows = H * sum(min(c["k"], n) for n in lens)
        return {"bytes": rows * (2 * (D + 2 * D) + 4), "flops": rows * 2 * D}
    first, _ = _ranges(c)
    seen = sum(lens) if first is None else sum(n - int(first[b, :new].min()) for b, (n, new) in enumerate(zip(lens, _new_lens(c))))
    return {"bytes": 2 * 2 * D * H * seen + sum(_new_lens(c)) * Hq * (4 * D + 4), "flops": 4 * D * Hq * _pairs(c)}


# ---- the same results in 64 bits ----------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    return {"append": _exact_append, "append8": _exact_append8, "attn8": _exact_attn8, "gather8": _exact_gather8, "prompt": _exact_prompt}[c["kind"]](s, c)


def _exact_rotation(s, c, b, i, row):
    """The matrix that turns token i of sequence b, float64 [D, D] (applied from the right)."""
    R = torch.eye(D, dtype=torch.float64, device="cuda")
    half = c["rot"] // 2
    t = s["table"][row].double()
    n = torch.arange(half, device="cuda")
    x, y = (2 * n, 2 * n + 1) if c["interleaved"] else (n, n + half)
    R[x, x], R[y, x], R[x, y], R[y, y] = t[:half], -t[half:], t[half:], t[:half]
    return R


def _exact_rows(s, c, b):
    """Turned q and k rows of sequence b, float64."""
    new, n = _new_lens(c)[b], _lens(c)[b]
    q, k = s["q"][b, :new].double(), s["k"][b, :new].double()
    if new <= 64:
        R = torch.stack([_exact_rotation(s, c, b, i, n - new + i) for i in range(new)])
        return torch.matmul(q, R), torch.matmul(k, R)
    # many tokens: as complex numbers
    half = c["rot"] // 2
    t = s["table"][n - new:n].double()[:, None]
    turn = torch.complex(t[..., :half].contiguous(), t[..., half:].contiguous())
    out = []
    for x in (q, k):
        r = x[..., :c["rot"]]
        z = torch.view_as_complex(r.reshape(*r.shape[:2], half, 2).contiguous()) if c["interleaved"] else torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous())
        z = z * turn
        r = torch.view_as_real(z).flatten(-2) if c["interleaved"] else torch.cat([z.real, z.imag], dim=-1)
        out.append(torch.cat([r, x[..., c["rot"]:]], dim=-1))
    return out


def _exact_append(s, c):
    q_out, K, V = s["q_out"].double(), s["K"].double(), s["V"].double()
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        q, k = _exact_rows(s, c, b)
        q_out[b, :new] = q
        K[b, :, n - new:n] = k.transpose(0, 1)
        V[b, :, n - new:n] = s["v"][b, :new].double().transpose(0, 1)
    return {"q": q_out, "K": K, "V": V}


def _exact_append8(s, c):
    blk, q_out = c["block"], s["q_out"].double()
    o = {n: s[n].double() for n in ("k8", "v8", "k_scale", "v_scale", "k_tail", "v_tail")}
    top = 448.0 if c["fmt"] == "e4m3" else 127.0
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        q, k = _exact_rows(s, c, b)
        q_out[b, :new] = q
        for x, name in ((k.to(torch.bfloat16).double(), "k"), (s["v"][b, :new].double(), "v")):
            x = x.transpose(0, 1)
            start = n - new
            from_tail = start % blk
            rows = torch.cat([o[name + "_tail"][b, :, :from_tail], x], dim=1)        # from row start - from_tail on
            base = start - from_tail
            full = (n - base) // blk
            for f in range(full):
                y = rows[:, f * blk:(f + 1) * blk]
                most = y.abs().amax(dim=(1, 2))
                scale = torch.exp2(torch.ceil(torch.log2(most / top) - 1e-12))
                y = y / scale[:, None, None]
                if c["fmt"] == "int8":
                    y = torch.round(y)
                else:                                    # 3 bits behind the leading one, down to steps of 2^-9
                    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)
                    y = torch.round(y / step) * step
                o[name + "8"][b, :, base + f * blk:base + (f + 1) * blk] = y
                o[name + "_scale"][b, :, base // blk + f] = scale
            left = rows[:, full * blk:]
            o[name + "_tail"][b, :, :left.shape[1]] = left
    return {"q": q_out, **o}


def _exact_row8(s, c, name, b, h, n):
    full = n // c["block"] * c["block"]
    x = s[name + "8"][b, h, :full].double() * s[name + "_scale"][b, h, :full // c["block"]].double().repeat_interleave(c["block"])[:, None]
    return torch.cat([x, s[name + "_tail"][b, h, :n - full].double()])


def _exact_attn8(s, c):
    G = c["hq"] // c["hkv"]
    out, lse = s["out"].double(), s["lse"].double()
    weights = None if s["weights"] is None else s["weights"].double()
    for b, n in enumerate(_lens(c)):
        for h in range(c["hkv"]):
            z = s["q"][b, h * G:(h + 1) * G].double() @ _exact_row8(s, c, "k", b, h, n).T * SCALE
            a = torch.softmax(z, dim=1)
            out[b, h * G:(h + 1) * G] = a @ _exact_row8(s, c, "v", b, h, n)
            lse[b, h * G:(h + 1) * G] = torch.logsumexp(z, dim=1)
            if weights is not None:
                weights[b, h * G:(h + 1) * G, :n] = a
    return {"out": out, "lse": lse, **({} if weights is None else {"weights": weights})}


def _exact_gather8(s, c):
    K, V = s["small_K"].double(), s["small_V"].double()
    for b, n in enumerate(_lens(c)):
        for h in range(c["hkv"]):
            at = s["idx"][b, h]
            at = at[at >= 0].long()
            K[b, h, :len(at)] = _exact_row8(s, c, "k", b, h, n)[at]
            V[b, h, :len(at)] = _exact_row8(s, c, "v", b, h, n)[at]
    return {"small_K": K, "small_V": V, "tail_start": s["seq_lens"]}


def _exact_prompt(s, c):
    G = c["hq"] // c["hkv"]
    out, lse = s["out"].double(), s["lse"].double()
    first, end = _ranges(c)
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        at = torch.arange(n - new, n, device="cuda")
        rows = torch.arange(n, device="cuda")
        lo = torch.zeros_like(at) if first is None else torch.from_numpy(first[b, :new]).cuda().long()
        hi = at + 1 if end is None else torch.from_numpy(end[b, :new]).cuda().long()
        seen = (rows >= lo[:, None]) & (rows < hi[:, None])
        far = (at[:, None] - rows).abs().double()
        for h in range(c["hq"]):
            z = s["q"][b, :new, h].double() @ s["K"][b, h // G, :n].double().T * SCALE
            if c["cap"]:
                z = torch.tanh(z / c["cap"]) * c["cap"]
            if s["slopes"] is not None:
                z = z - float(s["slopes"][h]) * far
            z = torch.where(seen, z, torch.full_like(z, -math.inf))
            lse[b, :new, h] = torch.logsumexp(z, dim=1)
            out[b, :new, h] = torch.softmax(z, dim=1) @ s["V"][b, h // G, :n].double()
    return {"out": out, "lse": lse}
