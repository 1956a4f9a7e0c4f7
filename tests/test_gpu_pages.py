"""rk_rope_append_paged, rk_page_scores, rk_page_select: refusals (no GPU needed), and against oracle/paged.py."""
import ctypes as C
import math
import sys

import numpy as np
import pytest
import torch

from oracle import paged as o
from oracle import new_tokens as nt

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


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().astype(np.int64) & 0xFFFF


def test_refusals_before_any_launch(rk):
    from paper_2411_05787_amd.binding import _Geom, _NewRows, _Pages, _Rope
    f, g = 0x10000, _Geom(2, 32, 8, 128, 0.1)
    P = lambda **k: _Pages(*[k.get(n, d) for n, d in (("k", f), ("v", f), ("k_min", f), ("k_max", f), ("sp", 8 * 32 * 128), ("sh", 32 * 128), ("n", 100), ("page", 32))])  # noqa: E731
    rows = _NewRows(f, f, f, 4096, 4096, 1024, 1024, 1024, 1024, 1)
    rope = _Rope(f, 100, 128, 0)

    def append(geom=g, r=rows, ro=rope, pages=None, table=f, width=128, sl=f, qo=f):
        return rk.lib.rk_rope_append_paged(C.byref(geom), C.byref(r), None if ro is None else C.byref(ro), None, C.byref(P() if pages is None else pages), table, width, sl, None,
                                           qo, None, 0, None)

    def scores(geom=g, q=f, sb=4096, st=4096, n=1, pages=None, table=f, width=128, sl=f, agg=0, s=f, ss=128):
        return rk.lib.rk_page_scores(C.byref(geom), q, sb, st, n, C.byref(P() if pages is None else pages), table, width, sl, None, agg, s, ss, None, 0, None)

    def select(geom=g, s=f, ss=128, n=1, page=32, sl=f, k=4, first=0, last=1, idx=f):
        return rk.lib.rk_page_select(C.byref(geom), s, ss, n, page, sl, None, k, first, last, idx, None, 0, None)

    for call in (append, scores):
        assert call(geom=_Geom(2, 72, 8, 128, 0.1)) == -2 and call(geom=_Geom(2, 33, 8, 128, 0.1)) == -1
        assert call(table=None) == -1 and call(table=f + 1) == -1 and call(width=0) == -1 and call(sl=None) == -1 and call(width=2 ** 27) == -2
        assert call(pages=P(page=8)) == -2 and call(pages=P(n=0)) == -1 and call(pages=P(k_max=None)) == -1 and call(pages=P(k_min=f + 4)) == -1
    assert append(pages=P(k=None)) == -1 and append(pages=P(sh=12)) == -1 and append(pages=P(sp=1 << 41)) == -2
    assert append(qo=None) == -1 and append(ro=None) == -1 and append(r=_NewRows(f, None, f, 0, 0, 0, 0, 0, 0, 1)) == -1
    assert append(r=_NewRows(f, f, f, 8192, 4096, 1024, 1024, 1024, 1024, 1)) == -1         # in place where q does not lie as q_out does
    assert scores(pages=P(k_min=None, k_max=None)) == -1 and scores(agg=3) == -2 and scores(s=None) == -1 and scores(ss=0) == -1 and scores(q=f + 8) == -1
    assert scores(n=0) == -1 and scores(sb=4) == -1
    assert select(s=None) == -1 and select(idx=None) == -1 and select(k=0) == -1 and select(first=-1) == -1 and select(last=-1) == -1 and select(page=24) == -2
    assert select(n=0) == -1 and select(ss=0) == -1 and select(n=2 ** 30) == -2 and select(geom=_Geom(2, 32, 8, 64, 0.1)) == -2


def test_refuses_counts_that_32_bits_do_not_step_past(rk):
    from paper_2411_05787_amd.binding import _Geom, _Pages
    f = 0x10000
    g, pages = _Geom(1, 1, 1, 128, 0.1), _Pages(f, f, f, f, 2048, 2048, 8, 16)

    def select(k, page=16):
        return rk.lib.rk_page_select(C.byref(g), f, 8, 1, page, f, None, k, 0, 1, f, None, 0, None)

    def scores(n):
        return rk.lib.rk_page_scores(C.byref(g), f, 0, 0, n, C.byref(pages), f, 8, f, None, 0, f, 8, None, 0, None)

    assert select(2 ** 31 - 1) == -2 and select(2 ** 27) == -2 and select(2 ** 24, 128) == -2
    assert scores(2 ** 30 + 1) == -2 and scores(2 ** 31 - 1) == -2


def test_the_oracle_orders_and_selects():
    x = np.array([0xFF80, 0x8000, 0x0000, 0x7F80, 0x7FC0, 0xFFC0, 0xBF80, 0x3F80])
    assert np.argsort(o.in_order(x)).tolist() == [5, 0, 6, 1, 2, 7, 3, 4]
    assert o.select([3.0, math.nan, 3.0, 5.0, 1.0, 9.0], 4, 3, 0, 0).tolist() == [0, 1, 3]
    assert o.select([3.0, 2.0, 3.0, 5.0, 1.0, 9.0], 4, 3, 2, 1).tolist() == [0, 1, 4] and o.select([1.0], 0, 3, 0, 1).tolist() == [0, -1, -1]
    assert o.select([1.0, 2.0], 5, 1, 0, 2).tolist() == [1] and o.select([1.0], -1, 2, 1, 1).tolist() == [-1, -1]


def tables(B, need, width, n_pages, seed=0):
    r = np.random.default_rng(seed)
    order, at = r.permutation(n_pages), 0
    t = np.full((B, width), -1, np.int64)
    for b, n in enumerate(need):
        t[b, :n] = order[at:at + n]
        at += n
    return t


APPEND = {
    # B, Hq, Hkv, T, lens, new, page, rot, interleaved
    "step": (1, 32, 8, 1, [2001], None, 16, 128, False),
    "step_first": (2, 8, 2, 1, [1, 17], None, 16, 128, True),
    "steps": (5, 28, 4, 1, [64, 65, 128, 1, 100], None, 64, 64, False),
    "idle": (3, 4, 1, 2, [40, 0, 33], [2, 0, 1], 32, 32, True),
    "drafted": (2, 7, 1, 5, [34, 130], [5, 3], 32, 96, False),
    "prompt": (1, 8, 2, 300, [300], None, 16, 128, False),
    "ragged_prompts": (4, 12, 4, 200, [200, 1, 0, 77], [200, 1, 0, 77], 128, 128, True),
    "chunk": (2, 16, 8, 70, [333, 129], [70, 65], 64, 16, False),
    "one_page": (1, 2, 2, 128, [128], None, 128, 128, False),
    "before_the_start": (1, 4, 2, 20, [12], None, 16, 128, False),               # 20 new tokens of a sequence of 12
    "negative": (2, 4, 2, 3, [-5, 30], [3, 3], 16, 128, False),
    "beyond_the_table": (1, 4, 2, 40, [100], None, 16, 128, False),              # a table of 5 pages
}


@gpu
@pytest.mark.parametrize("bounded", [True, False], ids=["bounds", "plain"])
@pytest.mark.parametrize("name", list(APPEND))
def test_append(rk, name, bounded):
    """The rows that rk_rope_append writes into a cache whose rows lie one behind the other, bit for bit; the bounds from the rows, exactly."""
    say("append", name)
    B, Hq, H, T, lens, new, page, rot, inter = APPEND[name]
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    width = 5 if name == "beyond_the_table" else max(1, -(-max(lens) // page)) + 1
    n_pages = B * width + 3
    table = tables(B, [width] * B, width, n_pages)
    if name == "chunk":
        table[0, 4], table[1, 1] = -1, n_pages                                    # rows of pages that are none are not written
    g = torch.Generator().manual_seed(3)
    w = torch.randn(B, T, Hq + 2 * H, 128, generator=g).to(torch.bfloat16).cuda()
    w[..., 3] = -0.0
    q, k, v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
    rope = rk.Rope(rk.rope_table(max(max(lens), 1) + 1, rot), interleaved=inter)
    old = torch.randn(n_pages, 2, H, page + 4, 128, generator=g).to(torch.bfloat16).cuda()       # a pool in parts of something larger
    K, V = old[:, 0, :, :page], old[:, 1, :, :page]
    before = old.clone()
    lo, hi = (torch.randn(n_pages, H, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    lo0, hi0 = lo.clone(), hi.clone()
    rows = width * page
    Kc, Vc = (torch.zeros(B, H, rows, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    qa, qb = (torch.full((B, T, Hq, 128), 5.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    nl = [T] * B if new is None else new
    rk.rk_rope_append(geom, q, k, v, rope, Kc, Vc, i32(lens), qa, new_lens=i32(new))
    rk.rk_rope_append_paged(geom, q, k, v, rope, rk.Pages(K, V, *((lo, hi) if bounded else ())), i32(table), i32(lens), qb, new_lens=i32(new))
    torch.cuda.synchronize()
    assert torch.equal(qa.view(torch.int16), qb.view(torch.int16))
    want, want_lo, want_hi = before.clone(), bits(lo0), bits(hi0)
    for b in range(B):
        start, stop = max(lens[b] - nl[b], 0), min(lens[b], rows)
        for j in range(start, stop):
            to = table[b, j // page]
            if 0 <= to < n_pages:
                want[to, 0, :, j % page], want[to, 1, :, j % page] = Kc[b, :, j], Vc[b, :, j]
        if nl[b] == 0 or stop <= start:
            continue
        for x in range(start // page, (stop - 1) // page + 1):
            to = table[b, x]
            if 0 <= to < n_pages:
                for h in range(H):
                    want_lo[to, h], want_hi[to, h] = o.bounds(bits(want[to, 0, h, :min(stop - x * page, page)]))
    assert torch.equal(old.view(torch.int16), want.view(torch.int16))
    if bounded:
        assert (bits(lo) == want_lo).all() and (bits(hi) == want_hi).all()


@gpu
def test_append_turns_as_the_formula_does(rk):
    """One token against fp64: cosines and sines rounded to fp32 (2^-24 each), two products and a sum in fp32, one rounding to bf16 (2^-8)."""
    geom = rk.Geom(1, 4, 2, 128, SCALE)
    g = torch.Generator().manual_seed(0)
    q, k, v = (torch.randn(1, 1, h, 128, generator=g).to(torch.bfloat16) for h in (4, 2, 2))
    rope = rk.Rope(rk.rope_table(600, 64))
    pool = rk.Pages.empty(geom, 40, 16)
    table = torch.arange(40, dtype=torch.int32, device="cuda").flip(0).view(1, 40).contiguous()
    out = torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    rk.rk_rope_append_paged(geom, q.cuda(), k.cuda(), v.cuda(), rope, pool, table, i32([501]), out)
    f = nt.rope_frequencies(64, 10000.0) * 500
    for x, y in ((q, out[0, 0]), (k, pool.k[39 - 31, :, 4])):
        want = nt.rope_turn(x[0, 0].double().numpy(), np.cos(f), np.sin(f), False)
        size = np.abs(x[0, 0].double().numpy()).max()
        assert (np.abs(y.double().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 6 * 2.0 ** -24 * size).all()
    assert torch.equal(pool.v[39 - 31, :, 4].cpu(), v[0, 0])


@gpu
def test_bounds_depend_on_the_rows_alone(rk):
    """Appended one at a time, in pieces and at once; with rows taken back and put again; with infinities, NaN and both zeros among the keys."""
    B, H, page, n = 1, 2, 32, 150
    geom = rk.Geom(B, 2, H, 128, SCALE)
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(B, n, H, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    k[0, 10, 0, 0], k[0, 11, 0, 1], k[0, 40, 1, 2], k[0, 41, 1, 2] = math.inf, math.nan, -math.inf, math.inf
    k[0, 64:96, 0, 5] = 0.0
    k[0, 70:80, 0, 5] = -0.0
    kb = k.view(torch.int16)
    kb[0, 100, 1, 7] = -1                                                         # a NaN with its sign set
    k, v = k.cuda(), v.cuda()
    table = torch.tensor([[4, 0, 3, 1, 2]], dtype=torch.int32, device="cuda")
    states = []
    for pieces in ([n], [1] * n, [31, 2, 31, 64, 22], [60, -7, 7, 90, -20, 20]):
        pool, at = rk.Pages.empty(geom, 5, page), 0
        for t in pieces:
            if t < 0:
                junk = torch.full((B, -t, H, 128), 50.0, dtype=torch.bfloat16, device="cuda")
                rk.rk_rope_append_paged(geom, None, junk, junk, None, pool, table, i32([at - 0]), None)      # (the last rows, written over)
                at += t
                continue
            rk.rk_rope_append_paged(geom, None, k[:, at:at + t], v[:, at:at + t], None, pool, table, i32([at + t]), None)
            at += t
        states.append([bits(x) for x in (pool.k, pool.v, pool.k_min, pool.k_max)])
        assert at == n
    for s in states[1:]:
        assert all((a == b).all() for a, b in zip(s, states[0]))
    for j, to in enumerate([4, 0, 3, 1, 2]):
        for h in range(H):
            lo, hi = o.bounds(states[0][0][to, h, :min(n - j * page, page)])
            assert (states[0][2][to, h] == lo).all() and (states[0][3][to, h] == hi).all()


SCORES = {
    # B, Hq, Hkv, T, lens, new, page, agg
    "step": (2, 32, 8, 1, [2000, 33], None, 16, "max"),
    "step_seven": (3, 28, 4, 1, [700, 1, 64], None, 64, "mean"),
    "one_head": (1, 4, 4, 3, [300], None, 32, "first"),
    "tokens": (2, 16, 2, 21, [500, 130], [21, 6], 16, "max"),
    "five": (1, 10, 2, 40, [1500], None, 128, "mean"),
    "three_first": (2, 6, 2, 5, [333, 0], [5, 0], 16, "first"),
    "prompt": (1, 7, 1, 200, [200], None, 16, "max"),
    "many_pages": (1, 8, 2, 2, [20000], None, 16, "max"),
    "many_sequences": (34, 8, 8, 1, [50 + 37 * b for b in range(34)], None, 16, "max"),
    "many_sequences_seven": (33, 56, 8, 3, [300 + 9 * b for b in range(33)], [b % 4 for b in range(33)], 32, "mean"),
    "many_sequences_tokens": (32, 16, 8, 16, [700 - 11 * b for b in range(32)], [16] * 31 + [0], 128, "first"),
    "many_sequences_drafts": (32, 24, 8, 7, [70 * b for b in range(32)], [min(7, 70 * b) for b in range(32)], 16, "max"),
    "both_many": (32, 16, 8, 17, [500] * 32, None, 16, "mean"),
}


@gpu
@pytest.mark.parametrize("name", list(SCORES))
def test_scores(rk, name):
    """256 products of bf16 are exact in fp32 and added in it: 256 * 2^-24 of their sizes, one rounding by the scale, and the mean's G + 1."""
    say("scores", name)
    B, Hq, H, T, lens, new, page, agg = SCORES[name]
    G, geom = Hq // H, rk.Geom(B, Hq, H, 128, SCALE)
    width = max(1, -(-max(lens) // page))
    n_pages = B * width + 2
    table = tables(B, [width] * B, width, n_pages)
    gone = [(0, 1), (B - 1, 0)] if width > 2 else []
    for x, (b, j) in enumerate(gone):
        table[b, j] = [-1, n_pages][x]
    g = torch.Generator().manual_seed(1)
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16)
    q[..., 7] = -0.0
    a, c = (torch.randn(n_pages, H, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    lo, hi = torch.minimum(a, c), torch.maximum(a, c)
    K = torch.zeros(n_pages, H, page, 128, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(B, T, Hq + 2, 128, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 1:1 + Hq] = q.cuda()
    for W in (width, width + 5, max(1, width - 1)):
        out = torch.full((B, T, H, W), 7.0, device="cuda")
        rk.rk_page_scores(geom, wide[:, :, 1:1 + Hq], rk.Pages(K, K, lo.cuda(), hi.cuda()), i32(table), i32(lens), out, new_lens=i32(new),
                          agg={"max": rk.RK_AGG_MAX, "mean": rk.RK_AGG_MEAN, "first": rk.RK_AGG_FIRST}[agg])
        got = out.double().cpu().numpy()
        nl = [T] * B if new is None else new
        for b in range(B):
            there = (table[b] >= 0) & (table[b] < n_pages)
            at = np.where(there, table[b], 0)
            for i in range(T):
                last = (lens[b] - nl[b] + i) // page if i < nl[b] else -1
                n = max(0, min(last + 1, width, W))
                assert (got[b, i, :, n:] == 7).all(), (name, b, i)
                for h in range(H):
                    want, size = o.page_scores(q[b, i, h * G:(h + 1) * G].double().numpy(), lo[at, h].double().numpy(), hi[at, h].double().numpy(), SCALE, agg)
                    ok = np.where(there[:n], np.abs(got[b, i, h, :n] - want[:n]) <= (256 + 1 + G + 1) * 2.0 ** -24 * size[:n], got[b, i, h, :n] == -math.inf)
                    assert ok.all(), (name, b, i, h)


@gpu
def test_scores_bound_what_the_rows_score_and_show_what_is_no_number(rk):
    B, Hq, H, page, n = 1, 8, 2, 16, 400
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(4)
    k = torch.randn(B, n, H, 128, generator=g).to(torch.bfloat16)
    k[0, 50, 0, 3], k[0, 100, 1, 4] = math.nan, math.inf
    pool = rk.Pages.empty(geom, 25, page)
    table = torch.arange(25, dtype=torch.int32, device="cuda").view(1, 25)
    rk.rk_rope_append_paged(geom, None, k.cuda(), k.cuda(), None, pool, table, i32([n]), None)
    q = torch.randn(B, 1, Hq, 128, generator=g).to(torch.bfloat16)
    out = torch.zeros(B, 1, H, 25, device="cuda")
    rk.rk_page_scores(geom, q.cuda(), pool, table, i32([n]), out)
    got = out.cpu().numpy()[0, 0]
    s = SCALE * np.einsum("hd,jgd->hgj", q[0, 0].double().numpy(), k[0].double().numpy())
    for h in range(H):
        top = s[h * 4:h * 4 + 4, h].max(axis=0).reshape(25, 16).max(axis=1)
        bad = np.isnan(got[h]) | (got[h] == math.inf)
        assert bad.tolist() == [j == (50 // 16 if h == 0 else 100 // 16) for j in range(25)]
        assert (got[h][~bad] >= top[~bad] - 1e-4).all()
    idx = torch.zeros(B, 1, H, 2, dtype=torch.int32, device="cuda")
    rk.rk_page_select(geom, out, page, i32([n]), 2, idx)
    assert idx.cpu().numpy()[0, 0].tolist() == [[3, 24], [6, 24]]


@gpu
@pytest.mark.parametrize("B,T,H,W,page,lens,new,k,first,last", [
    (1, 1, 1, 1, 16, [1], None, 1, 0, 1), (2, 1, 8, 64, 32, [2000, 77], None, 10, 1, 2), (1, 1, 2, 1024, 16, [16384], None, 64, 0, 0),
    (3, 5, 2, 40, 16, [640, 300, 9], [5, 3, 5], 7, 1, 1), (1, 40, 1, 313, 64, [20001], None, 40, 2, 3), (2, 1, 1, 9000, 16, [143999, 20000], None, 1000, 1, 1),
    (1, 2, 3, 10, 16, [500], None, 6, 0, 2), (2, 2, 1, 30, 128, [0, 3000], [0, 2], 100, 0, 1), (1, 3, 1, 20, 16, [2], [3], 4, 1, 0), (1, 1, 4, 257, 16, [4112], None, 256, 0, 0),
    (1, 1, 1, 100, 16, [1600], None, 3, 9, 9), (1, 1, 2, 33000, 16, [527999], None, 2000, 4, 4), (1, 3, 2, 65, 16, [1040], None, 64, 0, 0)])
@pytest.mark.parametrize("values", ["normal", "ties", "one", "special"])
def test_select(rk, B, T, H, W, page, lens, new, k, first, last, values):
    say("select", B, T, H, W, k, values)
    geom = rk.Geom(B, H, H, 128, 1.0)
    r = np.random.default_rng(W + k)
    x = r.standard_normal((B, T, H, W)).astype(np.float32)
    if values == "ties":
        x = np.round(x * 2) / 2 * np.where(r.random(x.shape) < 0.5, 1, -1).astype(np.float32)      # (both zeros)
    elif values == "one":
        x[:] = -3.25
    elif values == "special":
        for v in (math.nan, math.inf, -math.inf, 3e38, -3e38, 1e-42, -1e-42):
            x[r.random(x.shape) < 0.06] = v
    nl = [T] * B if new is None else new
    idx = torch.full((B, T, H, k), 77, dtype=torch.int32, device="cuda")
    rk.rk_page_select(geom, torch.from_numpy(x).cuda(), page, i32(lens), k, idx, new_lens=i32(new), keep_first=first, keep_last=last)
    got = idx.cpu().numpy()
    for b in range(B):
        assert (got[b, nl[b]:] == 77).all()
        for i in range(nl[b]):
            own = (lens[b] - nl[b] + i) // page
            for h in range(H):
                np.testing.assert_array_equal(got[b, i, h], o.select(x[b, i, h], own, k, first, last), err_msg=str((b, i, h)))


@gpu
@pytest.mark.parametrize("B,T,H,W", [(1, 200, 8, 700), (2, 513, 1, 1024), (1, 129, 8, 641), (1, 128, 8, 641), (3, 1, 4, 1024), (1, 1, 2, 640), (2, 3, 2, 1025), (1, 2, 1, 2048), (1, 2, 2, 2049), (2, 1, 1, 4096), (1, 1, 2, 4097)])
def test_select_in_many_and_few_rows(rk, B, T, H, W):
    say("select in rows", B, T, H, W)
    geom = rk.Geom(B, H, H, 128, 1.0)
    r = np.random.default_rng(W + T)
    x = np.round(r.standard_normal((B, T, H, W)) * 50).astype(np.float32)
    lens, idx = [W * 16 - 7 * b for b in range(B)], torch.full((B, T, H, 33), 77, dtype=torch.int32, device="cuda")
    rk.rk_page_select(geom, torch.from_numpy(x).cuda(), 16, i32(lens), 33, idx, keep_first=2, keep_last=2)
    got = idx.cpu().numpy()
    for b in range(B):
        for i in range(T):
            for h in range(H):
                np.testing.assert_array_equal(got[b, i, h], o.select(x[b, i, h], (lens[b] - T + i) // 16, 33, 2, 2), err_msg=str((b, i, h)))
