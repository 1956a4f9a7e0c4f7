"""Operators over a paged cache, timed: their plain forms in elementary torch operations, the calls that a program makes of
the library, what a pass cannot do without, and the same results in 64 bits.

  append  rotary positions of new tokens and their rows into pages, with each page's bounds of its keys (rk_rope_append_paged)
  paged   attention of new tokens over pages: a decode step's token, drafted ones, chunks of prompts (rk_paged_attn)
  prefix  the same for a batch whose sequences begin with the same rows, which are read once for all (rk_prefix_attn)
  score   a bound of every page's scores for each query, out of the page's bounds (rk_page_scores)
  select  the pages with the largest bounds (rk_page_select)
  sparse  attention over the rows of the pages that were selected for each token and KV head (rk_sparse_attn)

A cache is a pool of pages of 16 to 128 rows of every KV head, and a table that names the pages of each sequence in order; the pages
of a sequence lie anywhere in the pool.  Heads, lengths and batches are those of the benchmark's workloads (32 heads over 8 and 28 over 4,
2k to 128k rows, a ragged batch of 16), odd ones between them.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

D = 128
SCALE = float(np.float32(1.0 / math.sqrt(D)))


def _case(name, kind, **changes):
    c = {"kind": kind, "batch": 1, "hq": 32, "hkv": 8, "len": 2048, "min_len": 0, "new": 1, "page": 16, "shape": 1}
    c.update(changes)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # the smallest call: one new token of one sequence into its page, whose bounds are brought up to date; latency decides
        _case("append_step", "append", len=2001, rot=128, interleaved=False, bounds=True),
        # ragged prompts of a model that rotates half of the head, pairs side by side
        _case("append_prompts", "append", batch=5, hq=28, hkv=4, new=2048, min_len=300, page=64, rot=64, interleaved=True, bounds=True),
        # a served batch with ragged lengths, a token each, in small pages
        _case("paged_step16", "paged", batch=16, len=16384, min_len=4096, cap=0.0, window=0),
        # chunks of prompts behind what is cached already, capped scores, a sliding window
        _case("paged_chunk", "paged", batch=3, hq=28, hkv=4, new=700, len=9001, min_len=900, page=64, cap=30.0, window=4096),
        # a served batch behind one system prompt, a token each
        _case("prefix_step64", "prefix", batch=64, prefix=8192, len=8700, min_len=8212, page=32, cap=0.0),
        # drafted tokens of a few sequences that ask about one long document, of an odd length
        _case("prefix_drafts", "prefix", batch=6, hq=28, hkv=4, new=5, prefix=32777, len=34000, min_len=32900, cap=0.0),
        # bounds of all pages of a served batch for its tokens
        _case("score_step16", "score", batch=16, len=32768, min_len=8192, page=32, agg="max"),
        # ... for the tokens of a prompt's chunk
        _case("score_chunk", "score", hq=28, hkv=4, new=1000, len=20001, page=64, agg="mean"),
        # which pages a served batch reads at this step: the first, the last two and the best
        _case("select_step16", "select", batch=16, len=32768, min_len=8192, page=32, k=64, first=1, last=2),
        # ... every token of a chunk
        _case("select_chunk", "select", hq=28, hkv=4, new=1000, len=20001, page=64, k=40, first=1, last=1),
        # the step over 2048 rows of each
        _case("sparse_step16", "sparse", batch=16, len=32768, min_len=8192, page=32, k=64),
        # a chunk, each token over pages of its own
        _case("sparse_chunk", "sparse", hq=28, hkv=4, new=500, len=20001, page=64, k=32),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "paged", "paged", "prefix", "prefix", "score", "select", "sparse", "sparse"])
    hq, hkv = rng.choice([(32, 8), (32, 8), (28, 4), (28, 4), (8, 8), (16, 8), (64, 8), (20, 4), (5, 1)])
    c = _case(None, kind, hq=hq, hkv=hkv, page=rng.choice([16, 32, 64, 128]), shape=rng.randint(1, 10 ** 6))
    if kind == "append":
        c["new"] = rng.choice([1, _log_int(rng, 2, 8192)])
        c["batch"] = max(1, min(_log_int(rng, 1, 64), 8192 // c["new"]))
        c["rot"], c["interleaved"], c["bounds"] = rng.choice([128, 128, 64, 32, 96]), rng.random() < 0.4, rng.random() < 0.7
        c["len"] = c["new"] + rng.choice([0, _log_int(rng, 1, 2000)]) if c["new"] > 1 else _log_int(rng, 130, 4096)
    elif kind == "paged":
        c["batch"] = rng.choice([1, _log_int(rng, 2, 32)])
        c["len"] = min(_log_int(rng, 300, 131072), 131072 * 16 // (c["batch"] * hkv))
        c["new"] = rng.choice([1, 1, _log_int(rng, 2, 4096)])
        most = 3 * 700 * 9001 * 28                       # (query head, row) pairs of the largest case
        c["new"] = max(1, min(c["new"], c["len"], most // (c["batch"] * hq * c["len"])))
        c["cap"], c["window"] = rng.choice([0.0, 0.0, 20.0, 50.0]), rng.choice([0, 0, 500, 4096])
    elif kind == "prefix":
        c["batch"], c["prefix"] = _log_int(rng, 2, 64), _log_int(rng, 200, 32768)
        c["new"] = rng.choice([1, 1, rng.randint(2, 8)])
        c["batch"] = max(2, min(c["batch"], 64 * 32 * 8700 // (hq * c["new"] * c["prefix"])))
        c["len"] = c["prefix"] + _log_int(rng, c["new"], 2048)
        c["cap"] = rng.choice([0.0, 0.0, 30.0])
    else:
        c["batch"] = rng.choice([1, _log_int(rng, 2, 16)])
        c["len"] = min(_log_int(rng, 500, 131072), 131072 * 32 // (c["batch"] * hkv))
        c["new"] = rng.choice([1, 1, _log_int(rng, 2, 1000)])
        pages = -(-c["len"] // c["page"])
        if kind == "score":
            c["agg"] = rng.choice(["max", "max", "mean"])
            c["new"] = max(1, min(c["new"], c["len"], 1000 * 313 * 28 // (c["batch"] * hq * pages)))
        elif kind == "select":
            c["new"] = max(1, min(c["new"], c["len"], 1000 * 4 * 313 // (c["batch"] * hkv * pages)))
            c["k"], c["first"], c["last"] = max(4, min(1024, pages // rng.randint(2, 12))), rng.randint(0, 2), rng.randint(0, 2)
        else:
            c["k"] = max(4, min(1024, pages // rng.randint(4, 16)))
            c["new"] = max(1, min(c["new"], c["len"], 500 * 28 * 32 * 64 // (c["batch"] * hq * c["k"] * c["page"])))
    if c["batch"] > 1 and rng.random() < 0.7:
        low = c["prefix"] + c["new"] if kind == "prefix" else 1
        c["min_len"] = max(low, c["len"] // rng.randint(2, 6))
    return c


# ---- shapes, a function of the case alone -------------------------------------------------------

def _lens(c):
    """Rows of every sequence, the new tokens included (host numbers)."""
    n = int(c["len"])
    if not c["min_len"]:
        return [n] * c["batch"]
    r = random.Random(c["shape"])
    return [n] + [r.randint(min(c["min_len"], n), n) for _ in range(c["batch"] - 1)]


def _new_lens(c):
    return [min(int(c["new"]), n) for n in _lens(c)]


def _up(n, m):
    return (n + m - 1) // m * m


def _width(c):
    return _up(c["len"], c["page"]) // c["page"]


def _windowed(c):
    return bool(c.get("window"))


def _pairs(c):
    """(new token, row) pairs that the masks leave."""
    total = 0
    for n, new in zip(_lens(c), _new_lens(c)):
        p = np.arange(n - new, n)
        total += int((np.minimum(p + 1, c["window"]) if _windowed(c) else p + 1).sum())
    return total


# ---- inputs -------------------------------------------------------------------------------------

def _normal(g, *shape):
    return torch.randn(*shape, generator=g, device="cuda", dtype=torch.bfloat16)


def _int32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _table(c):
    """cos and sin of every position, fp32 [positions, rot]: the angles in 64 bits."""
    half = c["rot"] // 2
    f = 10000.0 ** (-torch.arange(half, dtype=torch.float64, device="cuda") / half)
    a = torch.arange(c["len"], dtype=torch.float64, device="cuda")[:, None] * f
    return torch.cat([a.cos(), a.sin()], dim=1).float()


def _pool(c, g, s):
    """Pages in any order, and the table: int32 [batch, width], -1 where a sequence has no page."""
    B, page, width = c["batch"], c["page"], _width(c)
    own_pages = [_up(n, page) // page for n in _lens(c)]
    shared = c.get("prefix", 0) // page                  # whole pages that all sequences name
    n_pages = shared + sum(n - shared for n in own_pages) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    at = shared
    for b, n in enumerate(own_pages):
        table[b, :shared] = order[:shared]
        table[b, shared:n] = order[at:at + n - shared]
        at += n - shared
    s["pages"] = table
    s["K"], s["V"] = _normal(g, n_pages, c["hkv"], page, D), _normal(g, n_pages, c["hkv"], page, D)
    if c.get("prefix", 0) % page:                        # the rows of the prefix in the page where it ends are everybody's
        a, first = c["prefix"] % page, table[0, shared].long()
        for n in ("K", "V"):
            s[n][table[:, shared].long(), :, :a] = s[n][first, :, :a].clone()
    if c["kind"] == "score" or c.get("bounds"):
        s["k_min"], s["k_max"] = s["K"].amin(dim=2), s["K"].amax(dim=2)


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    B, Hq, H, T = c["batch"], c["hq"], c["hkv"], c["new"]
    s = {"c": c, "seq_lens": _int32(_lens(c)), "new_lens": _int32(_new_lens(c))}
    if c["kind"] == "select":
        n = _width(c)
        # bounds grow towards the row's own place, and pages next to each other are alike
        x = torch.randn(B, T, H, n + 4, generator=g, device="cuda")
        s["scores"] = (3.0 * (x[..., :n] + x[..., 2:n + 2] + x[..., 4:]) + 2.0 * torch.arange(n, device="cuda") / n).contiguous()
        s["idx"] = torch.zeros(B, T, H, c["k"], dtype=torch.int32, device="cuda")
        return s
    _pool(c, g, s)
    if c["kind"] == "append":
        # the rows of one fused projection, as a layer has them
        qkv = _normal(g, B, T, Hq + 2 * H, D)
        s["q"], s["k"], s["v"] = qkv[:, :, :Hq], qkv[:, :, Hq:Hq + H], qkv[:, :, Hq + H:]
        s["table"] = _table(c)
        s["q_out"] = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
        return s
    gain = 4.0 if c.get("cap") else 1.0                  # scores that the cap bends
    s["q"] = (_normal(g, B, T, Hq, D).float() * gain).to(torch.bfloat16)
    if c["kind"] == "score":
        s["scores"] = torch.zeros(B, T, H, _up(_width(c), 64), device="cuda")
        return s
    s["out"] = torch.zeros(B, T, Hq, D, dtype=torch.bfloat16, device="cuda")
    s["lse"] = torch.zeros(B, T, Hq, device="cuda")
    s["first"] = None
    if _windowed(c):
        p = (s["seq_lens"] - s["new_lens"])[:, None] + torch.arange(T, device="cuda", dtype=torch.int32)
        s["first"] = (p + 1 - c["window"]).clamp(min=0).int().contiguous()
    if c["kind"] == "prefix":
        s["prefix_len"] = _int32([c["prefix"]])
        s["prefix_pages"] = s["pages"][0, :_up(c["prefix"], c["page"]) // c["page"]].contiguous()
    if c["kind"] == "sparse":                            # pages that a token sees, its own among them, in their order
        k = c["k"]
        s["idx"] = torch.full((B, T, H, k), -1, dtype=torch.int32, device="cuda")
        for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
            last = torch.arange(n - new, n, device="cuda") // c["page"]
            x = torch.rand(new, H, _width(c), generator=g, device="cuda")
            j = torch.arange(_width(c), device="cuda")
            x = torch.where(j > last[:, None, None], torch.full_like(x, -1.0), x)
            x = torch.where(j == last[:, None, None], torch.full_like(x, 2.0), x)
            kk = min(k, _width(c))
            top, at = x.sort(dim=-1, descending=True)
            at = torch.where(top[..., :kk] < 0, torch.full_like(at[..., :kk], _width(c)), at[..., :kk]).sort(dim=-1).values
            s["idx"][b, :new, :, :kk] = torch.where(at == _width(c), torch.full_like(at, -1), at).int()
    return s


# ---- one pass -----------------------------------------------------------------------------------

def run(s):
    return (_own if own else _plain)[s["c"]["kind"]](s)


def _places(s):
    """The new tokens' rows [B, T] and which of them there are."""
    i = torch.arange(s["c"]["new"], device="cuda")
    return (s["seq_lens"] - s["new_lens"])[:, None] + i, i < s["new_lens"][:, None]


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


def _plain_append(s):
    c, page = s["c"], s["c"]["page"]
    row, real = _places(s)
    t = s["table"][row.clamp(0, c["len"] - 1).long()][:, :, None]
    cos, sin = t[..., :c["rot"] // 2], t[..., c["rot"] // 2:]
    q, k = (_plain_rotate(s[n].float(), cos, sin, c) for n in ("q", "k"))
    s["q_out"][real] = q[real]
    b = torch.arange(c["batch"], device="cuda")[:, None].expand_as(row)[real]
    at = row[real].long()
    to = s["pages"][b, at // page].long()
    s["K"][to, :, at % page] = k[real]
    s["V"][to, :, at % page] = s["v"][real]
    if not c["bounds"]:
        return {"q": s["q_out"], "K": s["K"], "V": s["V"]}
    # the pages with new rows: bounds of the rows that they hold now
    start, n = s["seq_lens"] - s["new_lens"], s["seq_lens"]
    j = torch.arange(s["pages"].shape[1], device="cuda")
    touched = (j >= (start // page)[:, None]) & (j * page < n[:, None]) & (s["new_lens"] > 0)[:, None]
    tb, tj = torch.nonzero(touched, as_tuple=True)
    to = s["pages"][tb, tj].long()
    held = tj[:, None] * page + torch.arange(page, device="cuda") < n[tb][:, None]
    x = s["K"][to].float()
    s["k_min"][to] = x.masked_fill(~held[:, None, :, None], math.inf).amin(dim=2).to(torch.bfloat16)
    s["k_max"][to] = x.masked_fill(~held[:, None, :, None], -math.inf).amax(dim=2).to(torch.bfloat16)
    return {"q": s["q_out"], "K": s["K"], "V": s["V"], "k_min": s["k_min"], "k_max": s["k_max"]}


def _plain_rows(s, name):
    """A sequence's rows in their order, fp32 [B, H, rows, D]."""
    x = s[name][s["pages"].clamp(min=0).long()].float()
    B, W, H, page, _ = x.shape
    return x.permute(0, 2, 1, 3, 4).reshape(B, H, W * page, D)


def _plain_attention(s, seen=None):
    """seen [B, H, 1, T, rows] (or None): rows beside what the causal mask leaves."""
    c, B, Hq, H, T = s["c"], s["c"]["batch"], s["c"]["hq"], s["c"]["hkv"], s["c"]["new"]
    G = Hq // H
    k, v = _plain_rows(s, "K"), _plain_rows(s, "V")
    rows = k.shape[2]
    p, real = _places(s)
    j = torch.arange(rows, device="cuda")
    hidden = j > p[..., None]
    if s["first"] is not None:
        hidden = hidden | (j < s["first"][..., None])
    hidden = hidden[:, None, None]
    if seen is not None:
        hidden = hidden | ~seen
    q = s["q"].float().view(B, T, H, G, D).permute(0, 2, 3, 1, 4).reshape(B, H, G * T, D)
    sc = torch.matmul(q, k.transpose(2, 3)).view(B, H, G, T, rows) * SCALE
    if c.get("cap"):
        sc = c["cap"] * torch.tanh(sc / c["cap"])
    sc = sc.masked_fill(hidden, -math.inf)
    m = sc.amax(dim=-1, keepdim=True)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    w = torch.exp(sc - m)
    total = w.sum(dim=-1, keepdim=True)
    w = torch.where(total > 0, w / total, torch.zeros_like(w))
    out = torch.matmul(w.view(B, H, G * T, rows), v).view(B, H, G, T, D).permute(0, 3, 1, 2, 4).reshape(B, T, Hq, D)
    lse = (m + torch.log(total)).view(B, Hq, T).permute(0, 2, 1)
    s["out"].copy_(torch.where(real[..., None, None], out.to(torch.bfloat16), s["out"]))
    s["lse"].copy_(torch.where(real[..., None], lse, s["lse"]))
    return {"out": s["out"], "lse": s["lse"]}


def _plain_score(s):
    c, B, Hq, H, T = s["c"], s["c"]["batch"], s["c"]["hq"], s["c"]["hkv"], s["c"]["new"]
    q = s["q"].float().view(B, T, H, Hq // H, D).permute(0, 2, 1, 3, 4).reshape(B, H, -1, D)
    at = s["pages"].clamp(min=0).long()
    lo, hi = (s[n][at].float().permute(0, 2, 3, 1) for n in ("k_min", "k_max"))
    x = (torch.matmul(q.clamp(min=0), hi) + torch.matmul(q.clamp(max=0), lo)) * SCALE
    x = x.view(B, H, T, Hq // H, -1)
    x = (x.amax(dim=3) if c["agg"] == "max" else x.mean(dim=3)).permute(0, 2, 1, 3)
    p, real = _places(s)
    j = torch.arange(x.shape[-1], device="cuda")
    there = (real[..., None] & (j <= (p // c["page"])[..., None]))[:, :, None]
    now = s["scores"][..., :x.shape[-1]]
    now.copy_(torch.where(there, x, now))
    return {"scores": s["scores"]}


def _plain_select(s):
    c, k = s["c"], s["c"]["k"]
    p, real = _places(s)
    j = torch.arange(s["scores"].shape[-1], device="cuda")
    last = (p // c["page"])[:, :, None, None]
    x = torch.where((j < c["first"]) | (j > last - c["last"]), torch.full_like(s["scores"], math.inf), s["scores"])
    x = torch.where(j <= last, x, torch.full_like(x, -math.inf))
    top, at = x.sort(dim=-1, descending=True, stable=True)
    n = j.shape[0]
    at = torch.where(at <= last, at, torch.full_like(at, n))[..., :k]
    at = torch.cat([at, torch.full((*at.shape[:-1], max(0, k - n)), n, device="cuda")], dim=-1).sort(dim=-1).values
    at = torch.where(at == n, torch.full_like(at, -1), at).int()
    s["idx"].copy_(torch.where(real[:, :, None, None], at, s["idx"]))
    return {"idx": s["idx"]}


def _plain_sparse(s):
    c = s["c"]
    B, T, H, k = s["idx"].shape
    chosen = torch.zeros(B, T, H, _width(c) + 1, dtype=torch.bool, device="cuda")
    chosen.scatter_(3, torch.where(s["idx"] >= 0, s["idx"], torch.full_like(s["idx"], _width(c))).long(), True)
    return _plain_attention(s, chosen[..., :-1].permute(0, 2, 1, 3)[:, :, None].repeat_interleave(c["page"], dim=-1))


_plain = {"append": _plain_append, "paged": _plain_attention, "prefix": _plain_attention, "score": _plain_score, "select": _plain_select,
          "sparse": _plain_sparse}


def _handles(s):
    """What a program makes once and keeps: geometry, the rotary table's handle, the pool, the scratch."""
    if "geom" not in s:
        import paper_2411_05787_amd as rk
        c = s["c"]
        s["rk"], s["geom"] = rk, rk.Geom(c["batch"], c["hq"], c["hkv"], D, SCALE)
        if "table" in s:
            s["rope"] = rk.Rope(s["table"], interleaved=c["interleaved"])
        if "K" in s:
            s["pool"] = rk.Pages(s["K"], s["V"], s.get("k_min"), s.get("k_max"))
        if c["kind"] == "paged":
            s["ws"] = rk.PromptWorkspace(s["geom"], c["new"], c["len"])
        elif c["kind"] == "prefix":
            s["ws"] = rk.PrefixWorkspace(s["geom"], c["new"], c["prefix"], c["len"] - c["prefix"])
        elif c["kind"] == "sparse":
            s["ws"] = rk.SparseWorkspace(s["geom"], c["new"], c["k"], c["page"])
    return s["rk"], s["geom"]


def _own_append(s):
    rk, geom = _handles(s)
    rk.rk_rope_append_paged(geom, s["q"], s["k"], s["v"], s["rope"], s["pool"], s["pages"], s["seq_lens"], s["q_out"], new_lens=s["new_lens"])
    return {"q": s["q_out"], "K": s["K"], "V": s["V"], **({"k_min": s["k_min"], "k_max": s["k_max"]} if s["c"]["bounds"] else {})}


def _own_paged(s):
    rk, geom = _handles(s)
    rk.rk_paged_attn(geom, s["q"], s["pool"], s["pages"], s["seq_lens"], s["c"]["len"], s["out"], new_lens=s["new_lens"], first=s["first"],
                     cap=s["c"]["cap"], lse=s["lse"], workspace=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_prefix(s):
    rk, geom = _handles(s)
    c = s["c"]
    rk.rk_prefix_attn(geom, s["q"], s["pool"], s["prefix_pages"], s["prefix_len"], c["prefix"], s["pages"], s["seq_lens"], c["len"] - c["prefix"],
                      s["out"], new_lens=s["new_lens"], cap=c["cap"], lse=s["lse"], workspace=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


def _own_score(s):
    rk, geom = _handles(s)
    rk.rk_page_scores(geom, s["q"], s["pool"], s["pages"], s["seq_lens"], s["scores"], new_lens=s["new_lens"],
                      agg=rk.RK_AGG_MAX if s["c"]["agg"] == "max" else rk.RK_AGG_MEAN)
    return {"scores": s["scores"]}


def _own_select(s):
    rk, geom = _handles(s)
    c = s["c"]
    rk.rk_page_select(geom, s["scores"], c["page"], s["seq_lens"], c["k"], s["idx"], new_lens=s["new_lens"], keep_first=c["first"],
                      keep_last=c["last"])
    return {"idx": s["idx"]}


def _own_sparse(s):
    rk, geom = _handles(s)
    rk.rk_sparse_attn(geom, s["q"], s["pool"], s["pages"], s["idx"], s["seq_lens"], s["out"], new_lens=s["new_lens"], lse=s["lse"],
                      workspace=s["ws"])
    return {"out": s["out"], "lse": s["lse"]}


_own = {"append": _own_append, "paged": _own_paged, "prefix": _own_prefix, "score": _own_score, "select": _own_select, "sparse": _own_sparse}


# ---- what a pass cannot do without --------------------------------------------------------------

def work(c):
    lens, new_lens, Hq, H, page = _lens(c), _new_lens(c), c["hq"], c["hkv"], c["page"]
    n = sum(new_lens)
    ends = n * Hq * (4 * D + 4)                          # queries in, outputs and log-sum-exps out
    if c["kind"] == "append":
        rows = n * (2 * Hq + 4 * H) * D * 2 + n * c["rot"] * 4
        if c["bounds"]:                                  # bounds out, the rows that were in the first page already back in
            rows += sum(_up(m, page) // page - (m - new) // page for m, new in zip(lens, new_lens)) * H * 2 * D * 2
            rows += sum((m - new) % page for m, new in zip(lens, new_lens)) * H * D * 2
        return {"bytes": rows, "flops": n * (Hq + H) * 3 * c["rot"]}
    if c["kind"] == "paged":
        seen = sum(m - max(0, m - new + 1 - c["window"]) if _windowed(c) else m for m, new in zip(lens, new_lens))
        return {"bytes": 4 * D * H * seen + ends, "flops": 4 * D * Hq * _pairs(c)}
    if c["kind"] == "prefix":
        seen = c["prefix"] + sum(m - c["prefix"] for m in lens)
        return {"bytes": 4 * D * H * seen + ends, "flops": 4 * D * Hq * _pairs(c)}
    if c["kind"] in ("score", "select"):
        pages = [p // page + 1 for m, new in zip(lens, new_lens) for p in range(m - new, m)]
        if c["kind"] == "select":
            return {"bytes": 4 * H * (sum(pages) + n * c["k"]), "flops": H * sum(pages)}
        return {"bytes": 4 * D * H * sum(_up(m, page) // page for m in lens) + n * Hq * 2 * D + 4 * H * sum(pages), "flops": 4 * D * Hq * sum(pages)}
    most = c["k"] * page
    seen = sum(min(m, most * new) for m, new in zip(lens, new_lens))
    pairs = sum(min(p + 1, most) for m, new in zip(lens, new_lens) for p in range(m - new, m))
    return {"bytes": 4 * D * H * seen + ends + 4 * n * H * c["k"], "flops": 4 * D * Hq * pairs}


# ---- the same results in 64 bits ----------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    return {"append": _exact_append, "paged": _exact_attention, "prefix": _exact_attention, "score": _exact_score, "select": _exact_select,
            "sparse": _exact_attention}[c["kind"]](s, c)


def _exact_turned(x, s, c, first, n):
    """Rows of tokens first .. n - 1, [tokens, heads, D], as complex numbers that are turned."""
    half = c["rot"] // 2
    t = s["table"][first:n].double()[:, None]
    turn = torch.complex(t[..., :half].contiguous(), t[..., half:].contiguous())
    x = x.double()
    r = x[..., :c["rot"]]
    if c["interleaved"]:
        z = torch.view_as_complex(r.reshape(*r.shape[:2], half, 2).contiguous()) * turn
        r = torch.view_as_real(z).flatten(-2)
    else:
        z = torch.complex(r[..., :half].contiguous(), r[..., half:].contiguous()) * turn
        r = torch.cat([z.real, z.imag], dim=-1)
    return torch.cat([r, x[..., c["rot"]:]], dim=-1)


def _exact_append(s, c):
    page, pages = c["page"], s["pages"].cpu().numpy()
    o = {"q": s["q_out"].double(), "K": s["K"].double(), "V": s["V"].double()}
    if c["bounds"]:
        o["k_min"], o["k_max"] = s["k_min"].double(), s["k_max"].double()
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        start = n - new
        o["q"][b, :new] = _exact_turned(s["q"][b, :new], s, c, start, n)
        k = _exact_turned(s["k"][b, :new], s, c, start, n)
        for j in range(start // page, (n - 1) // page + 1):
            lo, hi = max(start, j * page), min(n, (j + 1) * page)
            to = int(pages[b, j])
            o["K"][to, :, lo - j * page:hi - j * page] = k[lo - start:hi - start].transpose(0, 1)
            o["V"][to, :, lo - j * page:hi - j * page] = s["v"][b, lo - start:hi - start].double().transpose(0, 1)
            if c["bounds"]:
                held = o["K"][to, :, :hi - j * page]
                o["k_min"][to], o["k_max"][to] = held.min(dim=1).values, held.max(dim=1).values
    return o


def _exact_attention(s, c):
    page, G = c["page"], c["hq"] // c["hkv"]
    out, lse = s["out"].double(), s["lse"].double()
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        mine = s["pages"][b, :_up(n, page) // page].long()
        at, rows = torch.arange(n - new, n, device="cuda"), torch.arange(n, device="cuda")
        seen = rows <= at[:, None]
        if _windowed(c):
            seen = seen & (rows > at[:, None] - c["window"])
        for g in range(c["hkv"]):
            k, v = (s[x][mine, g].reshape(-1, D)[:n].double() for x in ("K", "V"))
            mask = seen
            if c["kind"] == "sparse":
                mask = seen & (s["idx"][b, :new, g, :, None] == (torch.arange(len(mine), device="cuda"))).any(dim=1).repeat_interleave(page, dim=1)[:, :n]
            for h in range(g * G, (g + 1) * G):
                z = s["q"][b, :new, h].double() @ k.T * SCALE
                if c.get("cap"):
                    z = torch.tanh(z / c["cap"]) * c["cap"]
                z = torch.where(mask, z, torch.full_like(z, -math.inf))
                lse[b, :new, h] = torch.logsumexp(z, dim=1)
                out[b, :new, h] = torch.softmax(z, dim=1) @ v
    return {"out": out, "lse": lse}


def _exact_score(s, c):
    page, G = c["page"], c["hq"] // c["hkv"]
    scores = s["scores"].double()
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        mine = s["pages"][b, :_up(n, page) // page].long()
        lo, hi = s["k_min"][mine].double(), s["k_max"][mine].double()
        for i0 in range(0, new, 16):
            q = s["q"][b, i0:min(i0 + 16, new)].double()
            for g in range(c["hkv"]):
                x = q[:, g * G:(g + 1) * G, None]
                z = torch.maximum(x * lo[:, g], x * hi[:, g]).sum(dim=-1) * SCALE
                z = z.amax(dim=1) if c["agg"] == "max" else z.mean(dim=1)
                for i in range(z.shape[0]):
                    last = (n - new + i0 + i) // page
                    scores[b, i0 + i, g, :last + 1] = z[i, :last + 1]
    return {"scores": scores}


def _exact_select(s, c):
    idx, scores = s["idx"].cpu().numpy(), s["scores"].cpu().numpy().astype(np.float64)
    for b, (n, new) in enumerate(zip(_lens(c), _new_lens(c))):
        for i in range(new):
            last = (n - new + i) // c["page"]
            j = np.arange(last + 1)
            kept = (j < c["first"]) | (j > last - c["last"])
            for g in range(c["hkv"]):
                x = scores[b, i, g, :last + 1]
                best = np.sort(np.lexsort((j, -x, ~kept))[:c["k"]])
                idx[b, i, g] = -1
                idx[b, i, g, :len(best)] = best
    return {"idx": torch.from_numpy(idx).cuda()}
