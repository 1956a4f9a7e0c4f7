"""rk_paged_attn, rk_prefix_attn, rk_sparse_attn: refusals (no GPU needed), and against oracle/paged.py."""
import ctypes as C
import math
import sys

import numpy as np
import pytest
import torch

from oracle import paged as o

gpu = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def i32(x):
    return None if x is None else torch.as_tensor(np.asarray(x), dtype=torch.int32).cuda()


def test_refusals_before_any_launch(rk):
    from paper_2411_05787_amd.binding import _Geom, _Pages, _PromptScores
    f = 0x10000
    g = _Geom(2, 32, 8, 128, 0.1)
    P = lambda **k: _Pages(*[k.get(n, d) for n, d in (("k", f), ("v", f), ("k_min", None), ("k_max", None), ("sp", 8 * 32 * 128), ("sh", 32 * 128), ("n", 100), ("page", 32))])  # noqa: E731
    ws = {"paged": rk.rk_prompt_workspace_bytes(rk.Geom(2, 32, 8, 128, 0.1), 4, 4096),
          "prefix": rk.lib.rk_prefix_workspace_bytes(C.byref(g), 4, 4096, 1024), "sparse": rk.lib.rk_sparse_workspace_bytes(C.byref(g), 4, 64, 32)}

    def call(kind, geom=g, q=f, sb=4 * 4096, st=4096, n=4, pages=None, table=f, width=128, sl=f, max_len=4096, sc=None, out=f, w=0x100000, nb=None,
             pt=f, pw=128, pl=f, mp=4096, own=1024, idx=f, k=64):
        pages = P() if pages is None else pages
        a = (C.byref(geom), q, sb, st, n, C.byref(pages))
        z = (None if sc is None else C.byref(sc), out, None, None, 0, w, ws[kind] if nb is None else nb, None)
        if kind == "paged":
            return rk.lib.rk_paged_attn(*a, table, width, sl, None, max_len, *z)
        if kind == "prefix":
            return rk.lib.rk_prefix_attn(*a, pt, pw, pl, mp, table, width, sl, None, own, *z)
        return rk.lib.rk_sparse_attn(*a, table, width, idx, k, sl, None, *z)

    for kind in ws:
        bad = lambda **x: call(kind, **x)  # noqa: E731
        assert bad(geom=_Geom(2, 72, 8, 128, 0.1)) == -2 and bad(geom=_Geom(2, 32, 8, 96, 0.1)) == -2 and bad(geom=_Geom(2, 33, 8, 128, 0.1)) == -1
        assert bad(q=None) == -1 and bad(out=None) == -1 and bad(sl=None) == -1 and bad(n=0) == -1 and bad(table=None) == -1 and bad(width=0) == -1
        assert bad(q=f + 2) == -1 and bad(out=f + 8) == -1 and bad(sb=4) == -1 and bad(st=-8) == -1 and bad(table=f + 2) == -1
        assert bad(pages=P(k=None)) == -1 and bad(pages=P(v=f + 8)) == -1 and bad(pages=P(sp=-8)) == -1 and bad(pages=P(sh=4)) == -1 and bad(pages=P(n=0)) == -1
        assert bad(pages=P(k_min=f)) == -1 and bad(pages=P(page=48)) == -2 and bad(pages=P(page=256)) == -2 and bad(pages=P(sp=1 << 40)) == -2
        assert bad(width=2 ** 26) == -2                                           # rows beyond 32 bits
        for cap in (-1.0, math.nan, math.inf):
            assert bad(sc=_PromptScores(cap, None, None, None)) == -1
        assert bad(n=2 ** 30) == -2
        assert bad(w=None) == -3 and bad(w=0x100010) == -3 and bad(nb=1024) == -3
    assert call("paged", max_len=0) == -1
    for x in (dict(pt=None), dict(pw=0), dict(pl=None), dict(mp=0), dict(own=0)):
        assert call("prefix", **x) == -1
    assert call("sparse", idx=None) == -1 and call("sparse", k=0) == -1 and call("sparse", idx=f + 1) == -1 and call("sparse", k=2 ** 27) == -2


def test_workspaces_cover_every_smaller_call(rk):
    for g in (rk.Geom(1, 32, 8, 128, 0.1), rk.Geom(1, 1, 1, 128, 0.1), rk.Geom(64, 28, 4, 128, 0.1), rk.Geom(300, 2, 2, 128, 0.1)):
        c = C.byref(g.c())
        for f, last in ((rk.lib.rk_prefix_workspace_bytes, ((1, 200, 1000), (1, 129, 5000))), (rk.lib.rk_sparse_workspace_bytes, ((1, 3, 64, 1000), (16, 32, 64, 128)))):
            seen = {(n, a, b): f(c, n, a, b) for n in (1, 2, 5, 17, 600) for a in last[0] for b in last[1]}
            assert all(v > 0 for v in seen.values())
            for (n, a, b), v in seen.items():
                assert all(v <= w for (n2, a2, b2), w in seen.items() if n2 >= n and a2 >= a and b2 >= b)
        for bad in ((0, 1, 1), (1, 0, 1), (1, 1, 0)):
            assert rk.lib.rk_prefix_workspace_bytes(c, *bad) == 0
        assert rk.lib.rk_sparse_workspace_bytes(c, 1, 1, 48) == 0
    with pytest.raises(rk.RkError):
        rk.PrefixWorkspace(rk.Geom(1, 33, 8, 128, 0.1), 1, 1, 1)


def test_binding_refuses(rk):
    g = rk.Geom(1, 4, 2, 128, 0.1)
    x, t = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16), torch.zeros(1, 2, dtype=torch.int32)
    with pytest.raises(ValueError):
        rk.Pages(x, x)
    for n, page in ((0, 16), (4, 48)):
        with pytest.raises(ValueError):
            rk.Pages.empty(g, n, page, device="cpu")
    with pytest.raises(ValueError):
        rk.rk_paged_attn(g, x, None, t, torch.zeros(1, dtype=torch.int32), 1, x)
    with pytest.raises(ValueError):
        rk.rk_sparse_attn(g, x, x, t, t, torch.zeros(1, dtype=torch.int32), x)


# ---- inputs ----

def ranges(kind, B, T, lens, new, seed):
    """first, end int32 [B, T] (None: causal)."""
    if kind == "causal":
        return None, None
    r = np.random.default_rng(seed)
    first, end = np.zeros((B, T), np.int32), np.zeros((B, T), np.int32)
    for b in range(B):
        p = np.arange(lens[b] - new[b], lens[b])
        if kind == "docs":
            starts = np.unique(np.concatenate([[0], r.integers(0, lens[b], 5)]))
            f, e = starts[np.searchsorted(starts, p, side="right") - 1], p + 1
        elif kind == "window":
            f, e = p - 37, p + 1                                                 # (below 0 at the start)
        elif kind == "both_ways":
            f, e = np.zeros_like(p), np.full_like(p, 10 ** 9)                    # beyond the rows there are
        else:                                                                    # holes: some see nothing
            f = r.integers(-3, lens[b] + 3, len(p))
            e = f + r.integers(-2, 90, len(p))
        first[b, :new[b]], end[b, :new[b]] = f, e
    return first, end


class Inputs:
    """A pool with pages in any order, of which `missing` of each sequence are no pages; what no sequence has is NaN."""

    def __init__(self, B, Hq, H, T, lens, new, page, masks="causal", cap=0.0, slopes=False, missing=0, prefix=None, width=None, seed=3):
        g, r = torch.Generator().manual_seed(seed), np.random.default_rng(seed)
        self.B, self.Hq, self.H, self.T, self.G, self.lens, self.page, self.cap = B, Hq, H, T, Hq // H, lens, page, cap
        self.new_given, self.new = new, [T] * B if new is None else new
        self.width = width or max(1, -(-max(lens) // page))
        shared = 0 if prefix is None else prefix // page
        need = [max(0, min(-(-n // page), self.width)) for n in lens]
        self.n_pages = shared + sum(max(0, n - shared) for n in need) + 4
        order = r.permutation(self.n_pages)
        self.table, at = np.full((B, self.width), -1, np.int64), shared
        for b, n in enumerate(need):
            self.table[b, :shared] = order[:shared]
            m = max(0, n - shared)
            self.table[b, shared:shared + m] = order[at:at + m]
            at += m
        self.table[:, -1:] = np.where(self.table[:, -1:] < 0, self.n_pages + 7, self.table[:, -1:])      # (a number beyond the pool)
        for b in range(B):
            if missing:
                self.table[b, r.integers(0, max(1, need[b]), missing)] = [-1, self.n_pages, 2 ** 31 - 1][b % 3]
        self.K, self.V = (torch.full((self.n_pages, H, page, 128), math.nan, dtype=torch.bfloat16) for _ in range(2))
        for b in range(B):
            number, slot, there = o.places(self.table[b], page, self.n_pages, max(lens[b], 0))
            for x in (self.K, self.V):
                v = torch.randn(len(slot), H, 128, generator=g).to(torch.bfloat16)
                x[number[there], :, slot[there]] = v[torch.from_numpy(there)]
        self.prefix = prefix
        if prefix is not None:
            n = -(-prefix // page)
            self.prefix_table = order[:shared].tolist() + [at + 0] * 0
            if n > shared:                                                       # the page where it ends: one of its own, its first rows everybody's
                extra = order[at]
                self.prefix_table = np.append(order[:shared], extra)
                a = prefix % page
                for x in (self.K, self.V):
                    x[extra] = math.nan
                    x[extra, :, :a] = torch.randn(H, a, 128, generator=g).to(torch.bfloat16)
                    for b in range(B):
                        if shared < self.width and 0 <= self.table[b, shared] < self.n_pages:
                            x[self.table[b, shared], :, :a] = math.nan             # (nobody looks there)
            self.prefix_table = np.asarray(self.prefix_table, dtype=np.int64)
        self.q = (torch.randn(B, T, Hq, 128, generator=g) * (3.0 if cap else 1.0)).to(torch.bfloat16)
        self.first, self.end = ranges(masks, B, T, lens, self.new, seed)
        self.slopes = torch.exp2(-torch.arange(1, Hq + 1).float() * 6 / Hq) if slopes else None
        self.idx = None

    def choose(self, k, seed=5):
        """Pages for every token and KV head: any order, some that are none, some beyond the token's own."""
        r = np.random.default_rng(seed)
        self.idx = np.full((self.B, self.T, self.H, k), -1, np.int64)
        for b in range(self.B):
            for i in range(self.T):
                for g in range(self.H):
                    x = r.permutation(self.width)[:k]
                    self.idx[b, i, g, :len(x)] = x
                    self.idx[b, i, g, r.integers(0, k, 1)] = [-1, self.width, -5][(i + g) % 3]
        return self

    def rows(self, b, g):
        """K, V [rows, 128] in f64 and which rows there are."""
        n = min(max(self.lens[b], 0), self.width * self.page)
        number, slot, there = o.places(self.table[b], self.page, self.n_pages, n)
        if self.prefix is not None:
            pn, ps, pt = o.places(self.prefix_table, self.page, self.n_pages, min(n, self.prefix))
            number[:len(pn)], slot[:len(pn)], there[:len(pn)] = pn, ps, pt
        out = []
        for x in (self.K, self.V):
            v = x[np.where(there, number, 0), g, slot].double().numpy()
            v[~there] = math.nan
            out.append(v)
        return out[0], out[1], there

    def seen(self, b, i, g, there):
        p = self.lens[b] - self.new[b] + i
        lo, hi = (0, p + 1) if self.first is None else (int(self.first[b, i]), int(self.end[b, i]))
        j = np.arange(len(there))
        ok = there & (j >= lo) & (j < hi)
        if self.idx is not None:
            ok &= np.isin(j // self.page, self.idx[b, i, g])
        return p, j[ok]

    def device(self, rk, strided=True):
        """Pool, queries and the arguments that all calls share; the pool's pages and heads parts of something larger."""
        geom = rk.Geom(self.B, self.Hq, self.H, 128, SCALE)
        if strided:
            wide = torch.full((self.n_pages, 2, self.H, self.page + 8, 128), math.nan, dtype=torch.bfloat16, device="cuda")
            K, V = wide[:, 0, :, :self.page], wide[:, 1, :, :self.page]
            K.copy_(self.K.cuda())
            V.copy_(self.V.cuda())
            qw = torch.zeros(self.B, self.T, self.Hq + 3, 128, dtype=torch.bfloat16, device="cuda")
            q = qw[:, :, 1:1 + self.Hq]
            q.copy_(self.q.cuda())
        else:
            K, V, q = self.K.cuda(), self.V.cuda(), self.q.cuda()
        args = dict(new_lens=i32(self.new_given), first=i32(self.first), end=i32(self.end), cap=self.cap, slopes=None if self.slopes is None else self.slopes.cuda())
        return geom, rk.Pages(K, V), q, i32(self.table), i32(self.lens), args

    def blank(self):
        return (torch.full((self.B, self.T, self.Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((self.B, self.T, self.Hq), 9.0, device="cuda"))

    def check(self, out, lse, few, what):
        """Scores: 128 products added in fp32 and five roundings of the cap and the bias, 140 * 2^-24 of their terms' sizes and 2^-21 of the cap.
        Weights: twice that, 2^-20, 2^-22 of s - max; in the product with V 2^-8 where they are bf16 (not `few`), 2^-16 otherwise.  The output is rounded
        once, 2^-8."""
        a, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
        qf = self.q.double().numpy()
        for b in range(self.B):
            for g in range(self.H):
                K, V, there = self.rows(b, g)
                for i in range(self.new[b]):
                    p, seen = self.seen(b, i, g, there)
                    for h in range(g * self.G, (g + 1) * self.G):
                        at = (what, b, i, h)
                        s1 = 0.0 if self.slopes is None else float(self.slopes[h])
                        want, wl, s, size = o.attention(qf[b, i, h], K, V, seen, p, SCALE, self.cap, s1)
                        if not len(seen):
                            assert (a[b, i, h] == 0).all() and l[b, i, h] == -math.inf, at
                            continue
                        ds = 140 * 2.0 ** -24 * size.max() + 2.0 ** -21 * self.cap
                        w = np.exp(s - s.max())
                        w /= w.sum()
                        rel = 2 * ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(s - s.max()) + (2.0 ** -16 if few else 2.0 ** -8)
                        assert abs(l[b, i, h] - wl) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wl), (at, l[b, i, h], wl)
                        err = 2.0 ** -8 * np.abs(want) + (rel * w) @ np.abs(V[seen])
                        assert (np.abs(a[b, i, h] - want) <= err).all(), (at, np.abs(a[b, i, h] - want).max())
        for b in range(self.B):                                                  # entries that are none are left alone
            assert (a[b, self.new[b]:] == 9).all() and (l[b, self.new[b]:] == 9).all(), what


PAGED = {
    "step": dict(B=1, Hq=32, H=8, T=1, lens=[300], new=None, page=16),
    "step_first_token": dict(B=2, Hq=8, H=2, T=1, lens=[1, 0], new=[1, 0], page=32, slopes=True),
    "step_ragged_cap": dict(B=3, Hq=28, H=4, T=1, lens=[1000, 129, 5], new=None, page=64, cap=5.0, slopes=True),
    "step_window": dict(B=2, Hq=7, H=1, T=1, lens=[700, 33], new=None, page=16, masks="window"),
    "step_missing": dict(B=3, Hq=8, H=2, T=1, lens=[500, 333, 64], new=None, page=16, missing=3),
    "step_all_missing": dict(B=2, Hq=4, H=2, T=1, lens=[16, 300], new=None, page=16, missing=30),
    "step_big_pages": dict(B=2, Hq=16, H=2, T=1, lens=[1500, 128], new=None, page=128),
    "step_alone": dict(B=16, Hq=16, H=4, T=1, lens=[400, 1, 77, 160] * 4, new=None, page=16),
    "step_beyond_the_table": dict(B=1, Hq=2, H=1, T=1, lens=[200], new=None, page=32, width=4),
    "long_step": dict(B=1, Hq=2, H=2, T=1, lens=[9000], new=None, page=16, missing=2),
    "drafted": dict(B=2, Hq=16, H=4, T=4, lens=[260, 90], new=[4, 3], page=32),
    "drafted_holes": dict(B=1, Hq=5, H=1, T=3, lens=[200], new=None, page=16, masks="holes", cap=3.0, slopes=True),
    "drafted_16": dict(B=1, Hq=1, H=1, T=16, lens=[500], new=None, page=64, masks="docs"),
    "far_cap": dict(B=1, Hq=4, H=1, T=2, lens=[100], new=None, page=16, cap=1000.0),
    "seventeen_rows": dict(B=1, Hq=1, H=1, T=17, lens=[500], new=None, page=16),
    "whole_prompt": dict(B=1, Hq=8, H=2, T=150, lens=[150], new=None, page=16),
    "ragged_prompts": dict(B=4, Hq=12, H=4, T=200, lens=[200, 1, 0, 77], new=[200, 1, 0, 77], page=32, slopes=True),
    "chunk": dict(B=2, Hq=28, H=4, T=70, lens=[600, 333], new=[70, 65], page=64, cap=8.0),
    "chunk_docs": dict(B=2, Hq=8, H=1, T=130, lens=[400, 130], new=None, page=16, masks="docs"),
    "chunk_window": dict(B=1, Hq=3, H=1, T=300, lens=[300], new=None, page=128, masks="window"),
    "chunk_both_ways": dict(B=1, Hq=4, H=2, T=90, lens=[90], new=None, page=32, masks="both_ways", slopes=True),
    "chunk_holes": dict(B=2, Hq=8, H=8, T=100, lens=[260, 100], new=[100, 30], page=16, masks="holes"),
    "chunk_missing": dict(B=3, Hq=4, H=2, T=60, lens=[700, 333, 128], new=None, page=16, missing=4),
    "chunk_missing_big": dict(B=2, Hq=8, H=2, T=40, lens=[900, 300], new=None, page=128, missing=1, cap=20.0),
    "split_rows": dict(B=1, Hq=2, H=1, T=40, lens=[5000], new=None, page=16),
    "split_far_cap": dict(B=1, Hq=2, H=1, T=33, lens=[2500], new=None, page=32, masks="docs", cap=500.0),
    "beyond_the_table": dict(B=1, Hq=2, H=1, T=30, lens=[100], new=None, page=16, width=6),
    "step_negative": dict(B=3, Hq=4, H=2, T=1, lens=[-5, 40, -2 ** 31], new=None, page=16, slopes=True),
    "drafted_short": dict(B=2, Hq=4, H=1, T=4, lens=[2, 40], new=None, page=16),                    # more new tokens than rows
    "chunk_negative": dict(B=3, Hq=4, H=2, T=50, lens=[-2 ** 31, 20, 90], new=None, page=32, cap=3.0),
}


@gpu
@pytest.mark.parametrize("name", list(PAGED))
def test_paged(rk, name):
    say("paged", name)
    x = Inputs(**PAGED[name])
    geom, pages, q, table, lens, args = x.device(rk)
    out, lse = x.blank()
    args["workspace"] = rk.PromptWorkspace(geom, x.T, x.width * x.page)
    rk.rk_paged_attn(geom, q, pages, table, lens, x.width * x.page, out, lse=lse, **args)
    torch.cuda.synchronize()
    x.check(out, lse, x.T * x.G <= 16, name)
    geom, pages, q, table, lens, _ = x.device(rk, strided=False)
    again = torch.full_like(out, 9.0)
    rk.rk_paged_attn(geom, q, pages, table, lens, x.width * x.page, again, **args)
    assert torch.equal(out, again)


@gpu
def test_paged_wide_form(rk):
    """Two rounds of workgroups of 256 rows: 64 rows to a wavefront; against the same rows one behind the other, which share every step of it."""
    B, Hq, H, n = 8, 16, 8, 8192
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn(B, n, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    K, V = (torch.randn(B, H, n, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lens = i32([n, n - 1, 5000, n, 33, 4097, n, 8000])
    order = torch.randperm(B * n // 16, generator=g, device="cuda")
    pages = [torch.empty(B * n // 16, H, 16, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    for p, x in zip(pages, (K, V)):
        p[order] = x.view(B, H, n // 16, 16, 128).permute(0, 2, 1, 3, 4).reshape(-1, H, 16, 128)
    ws = rk.PromptWorkspace(geom, n, n)
    outs = [torch.zeros_like(q) for _ in range(2)]
    new = lens.clone()
    rk.rk_prompt_attn(geom, q, K, V, lens, n, outs[0], new_lens=new, workspace=ws)
    rk.rk_paged_attn(geom, q, rk.Pages(*pages), order.view(B, -1).int(), lens, n, outs[1], new_lens=new, workspace=ws)
    assert torch.equal(*outs)


SPARSE = {
    "step": dict(B=2, Hq=32, H=8, T=1, lens=[1000, 333], new=None, page=16, k=20),
    "step_odd": dict(B=3, Hq=7, H=1, T=1, lens=[500, 16, 1], new=None, page=16, k=7),
    "one_page": dict(B=2, Hq=8, H=2, T=1, lens=[300, 31], new=None, page=32, k=1),
    "more_than_there_are": dict(B=1, Hq=4, H=2, T=1, lens=[200], new=None, page=64, k=9),
    "tokens": dict(B=2, Hq=8, H=2, T=20, lens=[400, 130], new=[20, 7], page=16, k=8),
    "tokens_capped": dict(B=1, Hq=10, H=2, T=9, lens=[700], new=None, page=128, k=3, cap=4.0, slopes=True),
    "window": dict(B=1, Hq=4, H=1, T=30, lens=[600], new=None, page=32, k=10, masks="window"),
    "holes": dict(B=2, Hq=4, H=1, T=12, lens=[300, 40], new=[12, 12], page=16, k=9, masks="holes"),
    "missing": dict(B=2, Hq=8, H=4, T=3, lens=[800, 100], new=None, page=16, missing=5, k=16),
    "many": dict(B=1, Hq=1, H=1, T=2, lens=[9000], new=None, page=16, k=400),
    "beyond_the_table": dict(B=1, Hq=2, H=1, T=1, lens=[300], new=None, page=32, width=5, k=4),
    "no_tokens": dict(B=2, Hq=2, H=1, T=2, lens=[0, 40], new=[0, 2], page=32, k=2),
    "negative": dict(B=3, Hq=4, H=2, T=3, lens=[-9, 2, -2 ** 31], new=None, page=16, k=2),
    "eight_heads": dict(B=2, Hq=16, H=2, T=3, lens=[200, 190], new=None, page=16, k=5),
    "step_capped": dict(B=2, Hq=8, H=2, T=1, lens=[700, 90], new=None, page=16, k=9, cap=4.0),
    "step_far_cap": dict(B=1, Hq=7, H=1, T=1, lens=[900], new=None, page=32, k=6, cap=200.0),
    "step_biased": dict(B=1, Hq=16, H=4, T=1, lens=[1500], new=None, page=64, k=12, slopes=True),
    "few_of_many_pages": dict(B=2, Hq=8, H=2, T=2, lens=[2600, 1900], new=[2, 1], page=16, k=11, cap=150.0, slopes=True),
    "few_with_holes": dict(B=2, Hq=12, H=2, T=3, lens=[900, 850], new=None, page=16, k=4, masks="holes"),
    "few_missing": dict(B=2, Hq=8, H=4, T=2, lens=[800, 700], new=None, page=16, missing=5, k=7),
    "tokens_far_cap": dict(B=1, Hq=6, H=2, T=11, lens=[500], new=None, page=32, k=5, cap=300.0, slopes=True),
    "tokens_half_a_page": dict(B=1, Hq=8, H=1, T=4, lens=[1024], new=None, page=16, k=8),
}


@gpu
@pytest.mark.parametrize("name", list(SPARSE))
def test_sparse(rk, name):
    say("sparse", name)
    c = dict(SPARSE[name])
    k = c.pop("k")
    x = Inputs(**c).choose(k)
    geom, pages, q, table, lens, args = x.device(rk)
    out, lse = x.blank()
    rk.rk_sparse_attn(geom, q, pages, table, i32(x.idx), lens, out, lse=lse, workspace=rk.SparseWorkspace(geom, x.T, k, x.page), **args)
    torch.cuda.synchronize()
    x.check(out, lse, True, name)


PREFIX = {
    "steps": dict(B=8, Hq=32, H=8, T=1, lens=[700, 613, 640, 900, 601, 800, 777, 651], new=None, page=16, prefix=600),
    "two": dict(B=2, Hq=8, H=2, T=1, lens=[400, 300], new=None, page=32, prefix=256),
    "one_row": dict(B=2, Hq=4, H=4, T=1, lens=[100, 2], new=None, page=16, prefix=1),
    "whole": dict(B=3, Hq=8, H=2, T=2, lens=[200, 210, 202], new=None, page=64, prefix=200),
    "drafted": dict(B=6, Hq=28, H=4, T=5, lens=[1400, 1300, 1206, 1201, 1205, 1333], new=[5, 4, 5, 1, 5, 3], page=16, prefix=1200),
    "shorter_ones": dict(B=4, Hq=8, H=1, T=3, lens=[300, 100, 0, 3], new=[3, 3, 0, 3], page=16, prefix=130),
    "chunks": dict(B=3, Hq=6, H=2, T=60, lens=[500, 360, 361], new=[60, 60, 33], page=32, prefix=301),
    "chunks_inside": dict(B=2, Hq=4, H=2, T=50, lens=[320, 60], new=None, page=16, prefix=290),      # new tokens within the prefix's rows too
    "capped": dict(B=5, Hq=8, H=2, T=4, lens=[400] * 5, new=None, page=64, prefix=321, cap=6.0, slopes=True),
    "window": dict(B=5, Hq=8, H=2, T=4, lens=[500, 420, 333, 410, 405], new=None, page=16, prefix=400, masks="window"),
    "holes": dict(B=4, Hq=4, H=1, T=9, lens=[300] * 4, new=None, page=16, prefix=100, masks="holes"),
    "missing": dict(B=4, Hq=8, H=2, T=1, lens=[700, 600, 650, 555], new=None, page=16, prefix=512, missing=4),
    "many_rows": dict(B=70, Hq=8, H=1, T=1, lens=[300 + 3 * i for i in range(70)], new=None, page=32, prefix=300),
    "long": dict(B=3, Hq=2, H=2, T=1, lens=[9100, 9001, 9050], new=None, page=16, prefix=9000),
    "no_prefix": dict(B=2, Hq=4, H=2, T=1, lens=[100, 50], new=None, page=16, prefix=0),
    "both_ways": dict(B=3, Hq=4, H=2, T=20, lens=[200, 150, 120], new=None, page=16, prefix=90, masks="both_ways"),
    "documents": dict(B=6, Hq=4, H=1, T=7, lens=[200, 150, 120, 99, 200, 140], new=None, page=32, prefix=90, masks="docs", slopes=True),
    "negative": dict(B=3, Hq=4, H=2, T=2, lens=[-7, 150, -2 ** 31], new=None, page=16, prefix=90),
    "many_pairs": dict(B=80, Hq=16, H=8, T=1, lens=[100 + i for i in range(80)], new=None, page=16, prefix=100),
    "many_pairs_odd": dict(B=129, Hq=2, H=2, T=1, lens=[60 + 2 * i for i in range(129)], new=[i % 2 for i in range(129)], page=16, prefix=33),
}


@gpu
@pytest.mark.parametrize("name", list(PREFIX))
def test_prefix(rk, name):
    say("prefix", name)
    x = Inputs(**PREFIX[name])
    geom, pages, q, table, lens, args = x.device(rk)
    out, lse = x.blank()
    P = max(x.prefix, 1)
    own = max(1, max(x.lens) - x.prefix)
    pt = i32(x.prefix_table if len(x.prefix_table) else [-1])
    rk.rk_prefix_attn(geom, q, pages, pt, i32([x.prefix]), P, table, lens, own, out, lse=lse, workspace=rk.PrefixWorkspace(geom, x.T, P, own), **args)
    torch.cuda.synchronize()
    x.check(out, lse, x.B * x.T * x.G <= 16, name)


@gpu
def test_prefix_length_is_bounded(rk):
    """*prefix_len beyond max_prefix counts as that, a negative one as 0; max_own bounds the rows behind it."""
    x = Inputs(B=3, Hq=4, H=2, T=1, lens=[200, 150, 96], new=None, page=16, prefix=96)
    geom, pages, q, table, lens, args = x.device(rk)
    ws = rk.PrefixWorkspace(geom, 1, 96, 200)
    pt = i32(x.prefix_table)

    def run(value, most, own):
        out, lse = x.blank()
        rk.rk_prefix_attn(geom, q, pages, pt, i32([value]), most, table, lens, own, out, lse=lse, workspace=ws, **args)
        return out, lse
    for a, b in ((run(10 ** 9, 96, 200), run(96, 96, 200)), (run(-5, 96, 200), run(0, 96, 200)), (run(96, 80, 200), run(80, 96, 200))):
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    out, lse = run(96, 96, 30)                                                   # rows 126 and on are not seen
    args["end"] = i32([[min(n, 126)] for n in x.lens])
    args["first"] = i32([[0]] * 3)
    assert all(torch.equal(u, v) for u, v in zip((out, lse), run(96, 96, 200)))


@gpu
def test_a_page_chosen_twice_counts_twice(rk):
    x = Inputs(B=1, Hq=4, H=2, T=2, lens=[300], new=None, page=16).choose(6)
    x.idx[0, :, :, :] = np.array([3, 7, 3, 17, 3, 7])
    geom, pages, q, table, lens, args = x.device(rk)
    out, lse = x.blank()
    rk.rk_sparse_attn(geom, q, pages, table, i32(x.idx), lens, out, lse=lse, workspace=rk.SparseWorkspace(geom, 2, 6, 16), **args)
    for g in range(2):
        K, V, _ = x.rows(0, g)
        for i in range(2):
            seen = np.concatenate([np.arange(16 * j, 16 * j + 16) for j in (3, 7, 3, 17, 3, 7)])
            for h in (2 * g, 2 * g + 1):
                want, wl, s, size = o.attention(x.q[0, i, h].double().numpy(), K, V, seen, 298 + i, SCALE)
                # (as Inputs.check, with weights of at most 1 / 96 of each other's sum)
                assert abs(float(lse[0, i, h]) - wl) <= 140 * 2.0 ** -24 * size.max() + 2.0 ** -20 * (1 + abs(wl))
                assert np.abs(out[0, i, h].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + (2.0 ** -16 + 300 * 2.0 ** -24 * size.max()) * np.abs(V).max()
