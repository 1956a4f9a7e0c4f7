"""The calls over a cache in pages as a server makes them: a system prompt once, sequences behind it, decode steps over all rows and over chosen pages; captured,
on streams, over pools past 32 bits, with infinities and NaN planted, through either marshalling."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import paged as o
from test_gpu_paged_attn import SCALE, Inputs, PAGED, PREFIX, SPARSE, i32

gpu = pytest.mark.gpu
pytestmark = gpu


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def same(a, b):
    """Bit for bit (a NaN is a NaN: rows of a prefix's last page that nobody else has are NaN in these pools)."""
    return torch.equal(a.contiguous().view(torch.int16), b.contiguous().view(torch.int16))


def bf(*shape, fill=0.0):
    return torch.full(shape, fill, dtype=torch.bfloat16, device="cuda")


@pytest.mark.parametrize("page,prefix", [(16, 70), (32, 64), (64, 130)])
def test_a_served_run(rk, page, prefix):
    """A system prompt goes into its pages once; three sequences name them and go on with prompts of their own, then decode: the same outputs as over a cache
    whose rows lie one behind the other, with the prefix read once or by each, over all pages or all of them chosen."""
    say("served", page, prefix)
    B, Hq, H, G = 3, 8, 2, 4
    one, geom = rk.Geom(1, Hq, H, 128, SCALE), rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(11)
    rope = rk.Rope(rk.rope_table(512, 128))
    width, cap = 512 // page, 512
    pool = rk.Pages.empty(geom, B * width + 3, page)
    order = torch.randperm(pool.n_pages, generator=g)
    table = order[:B * width].view(B, width).int().cuda()
    whole = prefix // page
    table[1:, :whole] = table[0, :whole]
    K, V = bf(B, H, cap, 128), bf(B, H, cap, 128)

    def new(T, n):
        w = torch.randn(n, T, Hq + 2 * H, 128, generator=g).to(torch.bfloat16).cuda()
        return w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]

    q, k, v = new(prefix, 1)
    qo = bf(1, prefix, Hq, 128)
    rk.rk_rope_append_paged(one, q, k, v, rope, pool, table[:1], i32([prefix]), qo)
    for b in range(B):                                                           # rows one behind the other: everybody's own
        rk.rk_rope_append(one, None, k, v, rope, K[b:b + 1], V[b:b + 1], i32([prefix]), None)
        if prefix % page:                                                        # the page where the prefix ends: a copy of its own
            pool.k[table[b, whole].long()] = pool.k[table[0, whole].long()].clone()
            pool.v[table[b, whole].long()] = pool.v[table[0, whole].long()].clone()
    prefix_table = torch.cat([table[0, :whole], table[0, whole:whole + 1]]).contiguous()
    lens = np.full(B, prefix)
    pws, xws = rk.PromptWorkspace(geom, 80, cap), rk.PrefixWorkspace(geom, 80, prefix, cap)
    steps = [[80, 33, 1], [1, 0, 5]] + [[1, 1, 1]] * 6
    for step, counts in enumerate(steps):
        T = max(counts)
        q, k, v = new(T, B)
        lens = lens + counts
        sl, nl = i32(lens), i32(counts)
        qa, qb = bf(B, T, Hq, 128), bf(B, T, Hq, 128)
        rk.rk_rope_append(geom, q, k, v, rope, K, V, sl, qa, new_lens=nl)
        rk.rk_rope_append_paged(geom, q, k, v, rope, pool, table, sl, qb, new_lens=nl)
        assert torch.equal(qa, qb)
        outs = [(bf(B, T, Hq, 128, fill=9.0), torch.full((B, T, Hq), 9.0, device="cuda")) for _ in range(4)]
        rk.rk_prompt_attn(geom, qa, K, V, sl, cap, outs[0][0], new_lens=nl, lse=outs[0][1], workspace=pws)
        rk.rk_paged_attn(geom, qb, pool, table, sl, cap, outs[1][0], new_lens=nl, lse=outs[1][1], workspace=pws)
        rk.rk_prefix_attn(geom, qb, pool, prefix_table, i32([prefix]), prefix, table, sl, cap - prefix, outs[2][0], new_lens=nl, lse=outs[2][1], workspace=xws)
        scores = torch.zeros(B, T, H, width, device="cuda")
        rk.rk_page_scores(geom, qb, pool, table, sl, scores, new_lens=nl)
        idx = torch.full((B, T, H, width), -1, dtype=torch.int32, device="cuda")
        rk.rk_page_select(geom, scores, page, sl, width, idx, new_lens=nl)
        rk.rk_sparse_attn(geom, qb, pool, table, idx, sl, outs[3][0], new_lens=nl, lse=outs[3][1], workspace=rk.SparseWorkspace(geom, T, width, page))
        torch.cuda.synchronize()
        # weights as bf16 on the one side and to 2^-17 on the other, at most 2^-8 of the values' size twice, and half a step of the output's each
        top = float(V.double().abs().max())
        for x, (a, l) in enumerate(outs[1:]):
            for b in range(B):
                assert (a[b, counts[b]:] == 9).all() and (l[b, counts[b]:] == 9).all(), (step, x)
                d = (a[b, :counts[b]].double() - outs[0][0][b, :counts[b]].double()).abs()
                assert not len(d) or d.max() <= 4 * 2.0 ** -8 * top, (step, x, b, d.max())
                dl = (l[b, :counts[b]] - outs[0][1][b, :counts[b]]).abs()
                assert not len(dl) or dl.max() <= 1e-4, (step, x, b)
        # fewer pages: those with the largest scores, each token's own always, and the rows of these alone
        kk = 4
        few = torch.zeros(B, T, H, kk, dtype=torch.int32, device="cuda")
        rk.rk_page_select(geom, scores, page, sl, kk, few, new_lens=nl, keep_first=1, keep_last=1)
        a, l = bf(B, T, Hq, 128, fill=9.0), torch.full((B, T, Hq), 9.0, device="cuda")
        rk.rk_sparse_attn(geom, qb, pool, table, few, sl, a, new_lens=nl, lse=l, workspace=rk.SparseWorkspace(geom, T, kk, page))
        for b in range(B):
            for i in range(counts[b]):
                p = int(lens[b] - counts[b] + i)
                for h in range(H):
                    chosen = few[b, i, h].cpu().numpy()
                    assert p // page in chosen and 0 in chosen
                    np.testing.assert_array_equal(chosen, o.select(scores[b, i, h].cpu().numpy(), p // page, kk, 1, 1))
                    seen = np.array([j for j in range(p + 1) if j // page in chosen])
                    for x in range(h * G, (h + 1) * G):
                        want, wl, s, size = o.attention(qb[b, i, x].double().cpu().numpy(), K[b, h].double().cpu().numpy(), V[b, h].double().cpu().numpy(), seen, p, SCALE)
                        assert np.abs(a[b, i, x].double().cpu().numpy() - want).max() <= 2.0 ** -8 * np.abs(want).max() + 2.0 ** -13 * top
                        assert abs(float(l[b, i, x]) - wl) <= 1e-4


def attentions(rk, x, k=6):
    """The three attentions over one pool: callables of (out, lse), each with scratch of its own."""
    geom, pages, q, table, lens, args = x.device(rk)
    cap = x.width * x.page
    ws = rk.PromptWorkspace(geom, x.T, cap), rk.PrefixWorkspace(geom, x.T, max(x.prefix, 1), cap), rk.SparseWorkspace(geom, x.T, k, x.page)
    pt, pl, idx = i32(x.prefix_table), i32([x.prefix]), i32(x.idx)
    return geom, lens, {
        "paged": lambda out, lse, **m: rk.rk_paged_attn(geom, q, pages, table, lens, cap, out, lse=lse, workspace=ws[0], **{**args, **m}),
        "prefix": lambda out, lse, **m: rk.rk_prefix_attn(geom, q, pages, pt, pl, max(x.prefix, 1), table, lens, cap, out, lse=lse, workspace=ws[1], **{**args, **m}),
        "sparse": lambda out, lse, **m: rk.rk_sparse_attn(geom, q, pages, table, idx, lens, out, lse=lse, workspace=ws[2], **{**args, **m})}


@pytest.mark.parametrize("T", [1, 3, 40])
def test_predicates_and_streams(rk, T):
    x = Inputs(B=3, Hq=8, H=2, T=T, lens=[300, 200, 260], new=None, page=16, prefix=100)
    x.idx = None
    y = Inputs(B=3, Hq=8, H=2, T=T, lens=[300, 200, 260], new=None, page=16, prefix=100).choose(6)
    x.idx = y.idx
    geom, lens, calls = attentions(rk, x)
    pred = i32([1, 0, 1])
    for name, call in calls.items():
        full, lse = x.blank()
        call(full, lse)
        some, slse = x.blank()
        call(some, slse, pred=pred, pred_val=1)
        torch.cuda.synchronize()
        assert (some[1] == 9).all() and (slse[1] == 9).all(), name
        for b in (0, 2):
            assert same(some[b], full[b]) and same(slse[b], lse[b]), (name, b)
        # two streams at once, each with its own scratch; and a stream handed over
        streams, got = [torch.cuda.Stream() for _ in range(2)], []
        for s in streams:
            with torch.cuda.stream(s):
                c = attentions(rk, x)[2][name]
                a = x.blank()
                for _ in range(10):
                    c(*a)
                got.append(a)
        torch.cuda.synchronize()
        again = x.blank()
        call(*again, stream=streams[0])
        torch.cuda.synchronize()
        for a, l in got + [again]:
            assert same(a, full) and same(l, lse), name


def test_captured(rk):
    """Append, scores, selection and the three attentions in one graph; a second graph over the same scratch; replayed in turn with the lengths changed
    and eager calls between."""
    B, Hq, H, page, n = 2, 8, 2, 16, 400
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(4)
    width = n // page
    old = torch.randn(2, B * width + 2, H, page, 128, generator=g).to(torch.bfloat16).cuda()
    table = torch.randperm(B * width + 2, generator=g)[:B * width].view(B, width).int().cuda()
    table[1, :3] = table[0, :3]
    rope = rk.Rope(rk.rope_table(n, 128))
    prefix_len, lens = i32([40]), i32([300, 200])
    ws = rk.PromptWorkspace(geom, 4, n), rk.PrefixWorkspace(geom, 4, 48, n), rk.SparseWorkspace(geom, 4, 5, page)

    class State:
        def __init__(self, T, seed):
            w = torch.randn(B, T, Hq + 2 * H, 128, generator=torch.Generator().manual_seed(seed)).to(torch.bfloat16).cuda()
            self.q, self.k, self.v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
            self.pool = rk.Pages(old[0].clone(), old[1].clone(), old[0].amin(dim=2), old[0].amax(dim=2))
            self.qo, self.scores, self.idx = bf(B, T, Hq, 128), torch.zeros(B, T, H, width, device="cuda"), torch.zeros(B, T, H, 5, dtype=torch.int32, device="cuda")
            self.out, self.lse = [bf(B, T, Hq, 128) for _ in range(3)], [torch.zeros(B, T, Hq, device="cuda") for _ in range(3)]

        def run(self):
            rk.rk_rope_append_paged(geom, self.q, self.k, self.v, rope, self.pool, table, lens, self.qo)
            rk.rk_page_scores(geom, self.qo, self.pool, table, lens, self.scores)
            rk.rk_page_select(geom, self.scores, page, lens, 5, self.idx, keep_first=1)
            rk.rk_paged_attn(geom, self.qo, self.pool, table, lens, n, self.out[0], lse=self.lse[0], workspace=ws[0])
            rk.rk_prefix_attn(geom, self.qo, self.pool, table[0, :3], prefix_len, 48, table, lens, n, self.out[1], lse=self.lse[1], workspace=ws[1])
            rk.rk_sparse_attn(geom, self.qo, self.pool, table, self.idx, lens, self.out[2], lse=self.lse[2], workspace=ws[2])

        def all(self):
            return [self.pool.k, self.pool.v, self.pool.k_min, self.pool.k_max, self.qo, self.scores, self.idx, *self.out, *self.lse]

    eager, held = [State(1, 1), State(4, 2)], [State(1, 1), State(4, 2)]
    for s in eager + held:
        s.run()
    torch.cuda.synchronize()
    graphs = []
    for s in held:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            s.run()
    for a, b, p in ((300, 200, 40), (301, 201, 40), (400, 17, 16), (333, 1, 0), (5, 399, 48), (300, 200, 33)):
        lens.copy_(i32([a, b]))
        prefix_len.fill_(p)
        for s, graph in zip(held, graphs):
            graph.replay()
        for s in eager:
            s.run()
        for graph in graphs:                                                     # (again: the rows are there already)
            graph.replay()
        torch.cuda.synchronize()
        for s, e in zip(held, eager):
            for x, (u, v) in enumerate(zip(s.all(), e.all())):
                assert torch.equal(u.nan_to_num(7.0), v.nan_to_num(7.0)), (a, b, p, x)


@pytest.mark.parametrize("T", [1, 30])
def test_pools_past_32_bits(rk, T):
    """Pages whose places are beyond 2^32 elements, reached through strides: everything as in a small pool."""
    say("past 32 bits", T)
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("needs 24 GiB")
    x = Inputs(B=2, Hq=8, H=2, T=T, lens=[150, 90], new=None, page=16, prefix=50).choose(4)
    geom, pages, q, table, lens, args = x.device(rk)
    far = 2 ** 32 // (x.n_pages - 1) // 8 * 8 + 8                                # the last page starts behind 2^32 elements
    big = torch.empty((x.n_pages - 1) * far + x.H * x.page * 128, dtype=torch.bfloat16, device="cuda")
    size, stride = (x.n_pages, x.H, x.page, 128), (far, x.page * 128, 128, 1)
    k, v = (torch.randn(2, T, x.H, 128, generator=torch.Generator().manual_seed(s)).to(torch.bfloat16).cuda() for s in (1, 2))
    res = []
    for wide in (False, True):
        if wide:
            # (keys and values in one buffer: the values' heads behind the keys')
            both = big.as_strided((x.n_pages, x.H, x.page, 128), stride)
            K = both
            K.copy_(x.K.cuda())
            V2 = torch.empty_like(big).as_strided(size, stride)
            V2.copy_(x.V.cuda())
            pool = rk.Pages(K, V2, bf(x.n_pages, x.H, 128), bf(x.n_pages, x.H, 128))
        else:
            pool = rk.Pages(x.K.cuda(), x.V.cuda(), bf(x.n_pages, x.H, 128), bf(x.n_pages, x.H, 128))
        rk.rk_rope_append_paged(geom, None, k, v, None, pool, table, lens, None)
        outs = [x.blank() for _ in range(3)]
        cap = x.width * x.page
        rk.rk_paged_attn(geom, q, pool, table, lens, cap, *outs[0][:1], lse=outs[0][1], workspace=rk.PromptWorkspace(geom, T, cap), **args)
        rk.rk_prefix_attn(geom, q, pool, i32(x.prefix_table), i32([50]), 50, table, lens, cap, *outs[1][:1], lse=outs[1][1],
                          workspace=rk.PrefixWorkspace(geom, T, 50, cap), **args)
        rk.rk_sparse_attn(geom, q, pool, table, i32(x.idx), lens, *outs[2][:1], lse=outs[2][1], workspace=rk.SparseWorkspace(geom, T, 4, x.page), **args)
        torch.cuda.synchronize()
        res.append([pool.k.clone().contiguous(), pool.v.clone().contiguous(), pool.k_min, pool.k_max, *[y for z in outs for y in z]])
    for i, (a, b) in enumerate(zip(*res)):
        assert same(a, b), i


@pytest.mark.parametrize("kind,name", [("paged", "step"), ("paged", "step_window"), ("paged", "drafted"), ("paged", "chunk_docs"), ("paged", "chunk_window"), ("paged", "chunk_holes"),
                                       ("paged", "whole_prompt"), ("paged", "split_rows"), ("sparse", "tokens"), ("sparse", "window"), ("sparse", "holes"),
                                       ("prefix", "drafted"), ("prefix", "window"), ("prefix", "chunks"), ("prefix", "holes"), ("prefix", "steps"), ("prefix", "two")])
def test_rows_that_a_token_does_not_see_have_no_part(rk, kind, name):
    """Infinities and NaN planted in V and in one key: tokens that do not see them get what they get without; tokens that do see one get what comes of it."""
    say("planted", kind, name)
    c = dict({"paged": PAGED, "prefix": PREFIX, "sparse": SPARSE}[kind][name])
    k = c.pop("k", 0)
    x = Inputs(**c)
    if k:
        x.choose(k)
    r = np.random.default_rng(1)
    clean = x.K.clone(), x.V.clone()
    planted = []
    for b in range(x.B):
        if x.lens[b] < 3:
            continue
        first = x.prefix if x.prefix else 0                                      # (the prefix's rows are everybody's)
        for j in sorted(set(r.integers(first, max(x.lens[b], first + 1), 3).tolist()) | {x.lens[b] - 2}):
            if j >= x.lens[b]:
                continue
            n, s, there = o.places(x.table[b], x.page, x.n_pages, x.lens[b])
            g, d, v = int(r.integers(x.H)), int(r.integers(128)), [math.inf, -math.inf, math.nan][int(r.integers(3))]
            if there[j] and j >= first:
                x.V[n[j], g, s[j], d] = v
                planted.append((b, g, j, d, v))
    dirty = x.K, x.V
    outs = []
    for x.K, x.V in (clean, dirty):
        geom, pages, q, table, lens, args = x.device(rk, strided=False)
        out, lse = x.blank()
        cap = x.width * x.page
        if kind == "paged":
            rk.rk_paged_attn(geom, q, pages, table, lens, cap, out, lse=lse, workspace=rk.PromptWorkspace(geom, x.T, cap), **args)
        elif kind == "sparse":
            rk.rk_sparse_attn(geom, q, pages, table, i32(x.idx), lens, out, lse=lse, workspace=rk.SparseWorkspace(geom, x.T, k, x.page), **args)
        else:
            rk.rk_prefix_attn(geom, q, pages, i32(x.prefix_table), i32([x.prefix]), x.prefix, table, lens, cap, out, lse=lse,
                              workspace=rk.PrefixWorkspace(geom, x.T, x.prefix, cap), **args)
        outs.append((out.double().cpu().numpy(), lse.double().cpu().numpy()))
    assert planted
    (a, la), (c, lc) = outs
    for b in range(x.B):
        for g in range(x.H):
            there = x.rows(b, g)[2]
            for i in range(x.new[b]):
                seen = set(x.seen(b, i, g, there)[1].tolist())
                hs = slice(g * x.G, (g + 1) * x.G)
                assert (la[b, i, hs] == lc[b, i, hs]).all(), (name, b, i, g)
                want = a[b, i, hs].copy()
                for bb, gg, j, d, v in planted:
                    if bb == b and gg == g and j in seen:
                        want[:, d] += v
                # (weights in two parts: an infinity may come out as NaN)
                assert (np.isfinite(c[b, i, hs]) == np.isfinite(want)).all(), (name, b, i, g)
                np.testing.assert_array_equal(c[b, i, hs], np.where(np.isfinite(want), want, c[b, i, hs]), err_msg=str((name, b, i, g)))


@pytest.mark.parametrize("T,prefix", [(1, 40), (4, 40), (30, 200)])
def test_keys_that_are_no_number(rk, T, prefix):
    """A NaN among the prefix's keys reaches every token that sees it, and one among a sequence's own keys that sequence alone."""
    x = Inputs(B=3, Hq=4, H=2, T=T, lens=[300, 260, 280], new=None, page=16, prefix=prefix)
    n, s, _ = o.places(x.table[1], 16, x.n_pages, 260)
    x.K[n[225], 0, s[225], 3] = math.nan
    for planted in (False, True):
        if planted:
            x.K[x.prefix_table[1], 1, 2, 0] = math.nan
        geom, pages, q, table, lens, args = x.device(rk)
        out, lse = x.blank()
        rk.rk_prefix_attn(geom, q, pages, i32(x.prefix_table), i32([prefix]), prefix, table, lens, 300, out, lse=lse, workspace=rk.PrefixWorkspace(geom, T, prefix, 300), **args)
        got = torch.isnan(out).all(dim=-1).cpu().numpy()
        for b in range(3):
            for i in range(T):
                p = x.lens[b] - T + i
                assert got[b, i, 2:].all() == planted and got[b, i, :2].all() == (b == 1 and p >= 225), (b, i)


def test_scale_zero_and_negative(rk):
    """All rows alike, and the largest product weighing least, in every form."""
    for T in (1, 30):
        for scale in (0.0, -SCALE):
            x = Inputs(B=2, Hq=4, H=2, T=T, lens=[200, 190], new=None, page=16, prefix=70, missing=1).choose(9)
            x.idx, idx = None, x.idx
            geom, pages, q, table, lens, args = x.device(rk)
            geom = rk.Geom(2, 4, 2, 128, scale)
            for kind in ("paged", "prefix", "sparse"):
                out, lse = x.blank()
                x.idx = idx if kind == "sparse" else None
                if kind == "paged":
                    x2, x.prefix = x.prefix, None
                    rk.rk_paged_attn(geom, q, pages, table, lens, 208, out, lse=lse, workspace=rk.PromptWorkspace(geom, T, 208), **args)
                elif kind == "prefix":
                    rk.rk_prefix_attn(geom, q, pages, i32(x.prefix_table), i32([70]), 70, table, lens, 208, out, lse=lse, workspace=rk.PrefixWorkspace(geom, T, 70, 208), **args)
                else:
                    x2, x.prefix = x.prefix, None
                    rk.rk_sparse_attn(geom, q, pages, table, i32(idx), lens, out, lse=lse, workspace=rk.SparseWorkspace(geom, T, 9, 16), **args)
                got, gl = out.double().cpu().numpy(), lse.double().cpu().numpy()
                for b in range(2):
                    for g in range(2):
                        K, V, there = x.rows(b, g)
                        for i in range(T):
                            p, seen = x.seen(b, i, g, there)
                            for h in (2 * g, 2 * g + 1):
                                want, wl, _, _ = o.attention(x.q[b, i, h].double().numpy(), K, V, seen, p, scale)
                                if kind != "prefix" and np.isnan(V[seen]).any():
                                    continue                                     # (rows that are the prefix's in its own pages only)
                                if not len(seen):
                                    assert (got[b, i, h] == 0).all() and gl[b, i, h] == -math.inf
                                    continue
                                assert abs(gl[b, i, h] - wl) <= 1e-4 and np.abs(got[b, i, h] - want).max() <= 3 * 2.0 ** -8 * np.abs(V[seen]).max(), (kind, T, scale, b, i, h)
                if kind != "prefix":
                    x.prefix = x2


FORMS = {"plain": "", "no_lens": "", "strided": "", "wrong_shape": "append paged prefix scores select sparse", "wrong_type": "append paged prefix scores select sparse",
         "int_cap": "paged prefix sparse", "stream": ""}


@pytest.mark.parametrize("form", list(FORMS))
def test_either_marshalling(rk, form, monkeypatch):
    """The C++ marshalling takes what the common case is and leaves the rest to Python; both give the same results and refuse the same calls."""
    say("marshalling", form)
    B, T, page = 2, 3, 16
    x = Inputs(B=B, Hq=8, H=2, T=T, lens=[120, 90], new=None, page=page, prefix=40).choose(4)
    names = ("rk_rope_append_paged", "rk_paged_attn", "rk_prefix_attn", "rk_page_scores", "rk_page_select", "rk_sparse_attn")
    native = rk.binding._native
    stream = torch.cuda.Stream() if form == "stream" else None

    def run():
        geom, pages, q, table, lens, args = x.device(rk, strided=form == "strided")
        args["new_lens"] = None if form == "no_lens" else i32([T, 2])
        pool = rk.Pages(pages.k, pages.v, bf(x.n_pages, 2, 128), bf(x.n_pages, 2, 128))
        if form == "wrong_shape":
            table = table[:1]
        if form == "wrong_type":
            lens = lens.long()
        args["cap"] = 5 if form == "int_cap" else 0.0
        nl = args["new_lens"]
        gen = torch.Generator().manual_seed(3)
        kv = [torch.randn(B, T, 2, 128, generator=gen).to(torch.bfloat16).cuda() for _ in range(2)]
        outs = [x.blank() for _ in range(3)]
        scores, idx = torch.zeros(B, T, 2, x.width, device="cuda"), torch.zeros(B, T, 2, 4, dtype=torch.int32, device="cuda")
        qo = bf(B, T, 8, 128)
        rope = rk.Rope(rk.rope_table(128, 64), interleaved=True)
        cap = x.width * page
        ws = rk.PromptWorkspace(geom, T, cap), rk.PrefixWorkspace(geom, T, 40, cap), rk.SparseWorkspace(geom, T, 4, page)
        pt, pl, ix = i32(x.prefix_table), i32([40]), i32(x.idx)
        wrong = form == "wrong_shape"
        torch.cuda.synchronize()
        res = {}
        for name, call in (
                ("append", lambda: rk.rk_rope_append_paged(geom, q, *kv, rope, pool, table, lens, qo, new_lens=nl, stream=stream)),
                ("paged", lambda: rk.rk_paged_attn(geom, q, pool, table, lens, cap, outs[0][0], lse=outs[0][1], workspace=ws[0], stream=stream, **args)),
                ("prefix", lambda: rk.rk_prefix_attn(geom, q, pool, pt, pl, 40, table, lens, cap, outs[1][0], lse=outs[1][1], workspace=ws[1], stream=stream, **args)),
                ("scores", lambda: rk.rk_page_scores(geom, q, pool, table, lens, scores, new_lens=nl, stream=stream)),
                ("select", lambda: rk.rk_page_select(geom, scores, page, lens, 3 if wrong else 4, idx, new_lens=nl, stream=stream)),
                ("sparse", lambda: rk.rk_sparse_attn(geom, q, pool, table, ix, lens, outs[2][0], lse=outs[2][1], workspace=ws[2], stream=stream, **args))):
            try:
                call()
                res[name] = None
            except (ValueError, TypeError) as e:
                res[name] = str(e)
        torch.cuda.synchronize()
        return res, [pool.k, pool.v, pool.k_min, pool.k_max, qo, scores, idx, *[y for z in outs for y in z]]

    taken = []

    def watched(call):
        def f(*a):
            taken.append(call(*a) is not None)
            return 0 if taken[-1] else None
        return f
    monkeypatch.setattr(rk.binding, "_native", type("watched", (), {n: staticmethod(watched(getattr(native, n))) for n in names}))
    by_cpp = run()
    monkeypatch.setattr(rk.binding, "_native", type("none", (), {n: staticmethod(lambda *a: None) for n in names}))
    by_python = run()
    assert by_cpp[0] == by_python[0], (by_cpp[0], by_python[0])
    assert [n for n, t in zip(by_cpp[0], taken) if not t] == FORMS[form].split() and len(taken) == 6
    assert all(by_cpp[0].values()) == (form in ("wrong_shape", "wrong_type"))
    for a, b in zip(by_cpp[1], by_python[1]):
        assert torch.equal(a.nan_to_num(3.0), b.nan_to_num(3.0))


def test_binding_refuses(rk):
    x = Inputs(B=2, Hq=4, H=2, T=2, lens=[40, 30], new=None, page=16, prefix=16).choose(2)
    geom, pages, q, table, lens, _ = x.device(rk)
    out, _ = x.blank()
    ws, xws, sws = rk.PromptWorkspace(geom, 2, 48), rk.PrefixWorkspace(geom, 2, 16, 48), rk.SparseWorkspace(geom, 2, 2, 16)
    pt, pl, idx = i32(x.prefix_table), i32([16]), i32(x.idx)
    bad = [lambda: rk.Pages(pages.k, pages.v[:, :1]), lambda: rk.Pages(pages.k[..., :64], pages.v[..., :64]), lambda: rk.Pages(pages.k, pages.v, bf(x.n_pages, 2, 128)),
           lambda: rk.Pages(pages.k, pages.v, bf(x.n_pages, 2, 64), bf(x.n_pages, 2, 64)), lambda: rk.Pages(pages.k.float(), pages.v.float()),
           lambda: rk.rk_paged_attn(rk.Geom(2, 4, 4, 128, 0.1), q, pages, table, lens, 48, out, workspace=ws),       # a pool of other heads
           lambda: rk.rk_paged_attn(geom, q, pages, table, lens, 49, out, workspace=ws), lambda: rk.rk_paged_attn(geom, q, pages, table.long(), lens, 48, out, workspace=ws),
           lambda: rk.rk_paged_attn(geom, q, pages, table[:, ::2], lens, 16, out, workspace=ws), lambda: rk.rk_paged_attn(geom, q, pages, table.cpu(), lens, 48, out, workspace=ws),
           lambda: rk.rk_prefix_attn(geom, q, pages, pt, pl, 16, table, lens, 48, out), lambda: rk.rk_prefix_attn(geom, q, pages, pt, pl, 17, table, lens, 48, out, workspace=xws),
           lambda: rk.rk_prefix_attn(geom, q, pages, pt.view(1, -1), pl, 16, table, lens, 48, out, workspace=xws),
           lambda: rk.rk_prefix_attn(geom, q, pages, pt, i32([16, 16]), 16, table, lens, 48, out, workspace=xws),
           lambda: rk.rk_page_scores(geom, q, pages, table, lens, torch.zeros(2, 2, 2, 3, device="cuda")),           # a pool without bounds
           lambda: rk.rk_page_select(geom, torch.zeros(2, 2, 3, device="cuda"), 16, lens, 2, idx), lambda: rk.rk_page_select(geom, torch.zeros(2, 2, 2, 3, device="cuda"), 16, lens, 3, idx),
           lambda: rk.rk_sparse_attn(geom, q, pages, table, idx[0], lens, out, workspace=sws), lambda: rk.rk_sparse_attn(geom, q, pages, table, idx[:, :1], lens, out, workspace=sws)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    for call in (lambda: rk.rk_page_select(geom, torch.zeros(2, 2, 2, 3, device="cuda"), 48, lens, 2, idx), lambda: rk.rk_prefix_attn(geom, q, pages, pt, pl, 16, table, lens, 0, out, workspace=xws),
                 lambda: rk.rk_paged_attn(geom, q, pages, table, lens, 0, out, workspace=ws)):
        with pytest.raises(rk.RkError):
            call()
