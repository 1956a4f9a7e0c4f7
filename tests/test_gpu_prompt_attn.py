"""rk_prompt_attn: refusals (no GPU needed), and against oracle/new_tokens.py."""
import ctypes as C
import math
import sys

import numpy as np
import pytest
import torch

import gen
from oracle import new_tokens as o

gpu = pytest.mark.gpu


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def test_refusals_before_any_launch(rk):
    from paper_2411_05787_amd.binding import _Geom, _Kv, _PromptScores
    g, f = _Geom(2, 32, 8, 128, 0.1), 0x10000
    kv = _Kv(f, f, 8 * 4096 * 128, 4096 * 128, 4096)
    nb = rk.rk_prompt_workspace_bytes(rk.Geom(2, 32, 8, 128, 0.1), 4, 4096)

    def attn(geom=g, q=f, sb=4 * 4096, st=4096, n=4, c=kv, sl=f, max_len=4096, sc=None, out=f, ws=0x100000, nb=nb):
        return rk.lib.rk_prompt_attn(C.byref(geom), q, sb, st, n, c, sl, None, max_len, None if sc is None else C.byref(sc), out, None, None, 0, ws, nb, None)

    assert attn(geom=_Geom(2, 72, 8, 128, 0.1)) == -2 and attn(geom=_Geom(2, 32, 8, 96, 0.1)) == -2 and attn(geom=_Geom(2, 33, 8, 128, 0.1)) == -1
    assert attn(q=None) == -1 and attn(out=None) == -1 and attn(sl=None) == -1 and attn(n=0) == -1 and attn(max_len=0) == -1
    assert attn(q=f + 2) == -1 and attn(out=f + 8) == -1 and attn(sb=4) == -1 and attn(st=-8) == -1
    assert attn(c=_Kv(f, None, 0, 0, 4096)) == -1 and attn(c=_Kv(f + 2, f, 0, 0, 4096)) == -1
    for cap in (-1.0, math.nan, math.inf):
        assert attn(sc=_PromptScores(cap, None, None, None)) == -1
    assert attn(n=2 ** 30) == -2
    assert attn(ws=None) == -3 and attn(ws=0x100010) == -3 and attn(nb=1024) == -3


def test_workspace_covers_every_smaller_call(rk):
    """rk_prompt_workspace_bytes(n, L) is enough for any call of up to n tokens and L rows: it only grows with both."""
    for g in (rk.Geom(1, 32, 8, 128, 0.1), rk.Geom(1, 1, 1, 128, 0.1), rk.Geom(3, 28, 4, 128, 0.1), rk.Geom(300, 2, 2, 128, 0.1)):
        last = 0
        for n in (1, 2, 3, 4, 5, 16, 17, 100, 1000, 8192):
            row = [rk.rk_prompt_workspace_bytes(g, n, m) for m in (1, 100, 128, 129, 5000, 131072)]
            assert row == sorted(row) and row[-1] >= last
            last = row[-1]
    with pytest.raises(rk.RkError):
        rk.rk_prompt_workspace_bytes(rk.Geom(1, 32, 8, 128, 0.1), 0, 10)


def test_binding_refuses(rk):
    g = rk.Geom(1, 4, 2, 128, 0.1)
    x = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rk.rk_prompt_attn(g, x, x, x, torch.zeros(1, dtype=torch.int32), 1, x)


def ranges(kind, B, T, lens, new, seed):
    """first, end int32 [B, T] (None: causal)."""
    if kind == "causal":
        return None, None
    r = np.random.default_rng(seed)
    first, end = np.zeros((B, T), np.int32), np.zeros((B, T), np.int32)
    for b in range(B):
        p = np.arange(lens[b] - new[b], lens[b])
        if kind in ("docs", "docs_prefix"):
            starts = np.unique(np.concatenate([[0], r.integers(0, lens[b], 5)]))
            w = np.searchsorted(starts, p, side="right") - 1
            f, e = starts[w], p + 1
            if kind == "docs_prefix":
                e = np.maximum(e, np.minimum(f + 20, np.append(starts[1:], lens[b])[w]))
        elif kind == "window":
            f, e = p - 9, p + 1                                                  # (below 0 at the start)
        elif kind == "both_ways":
            f, e = np.zeros_like(p), np.full_like(p, 10 ** 9)                     # beyond the rows there are
        else:                                                                    # holes: some see nothing
            f = r.integers(-3, lens[b] + 3, len(p))
            e = f + r.integers(-2, 90, len(p))
        first[b, :new[b]], end[b, :new[b]] = f, e
    return first, end


CASES = [
    # name, B, Hq, Hkv, n_new, lens, new_lens, masks, cap, slopes
    ("step", 1, 32, 8, 1, [300], None, "causal", 0.0, False),
    ("step_first_token", 2, 8, 2, 1, [1, 0], [1, 0], "causal", 0.0, True),
    ("step_ragged_cap", 3, 28, 4, 1, [1000, 129, 5], None, "causal", 5.0, True),
    ("step_window", 2, 7, 1, 1, [700, 33], None, "window", 0.0, False),
    ("drafted", 2, 16, 4, 4, [260, 90], [4, 3], "causal", 0.0, False),
    ("drafted_holes", 1, 5, 1, 3, [200], None, "holes", 3.0, True),
    ("drafted_16", 1, 1, 1, 16, [500], None, "docs", 0.0, False),
    ("seventeen_rows", 1, 1, 1, 17, [500], None, "causal", 0.0, False),
    ("whole_prompt", 1, 8, 2, 150, [150], None, "causal", 0.0, False),
    ("ragged_prompts", 4, 12, 4, 200, [200, 1, 0, 77], [200, 1, 0, 77], "causal", 0.0, True),
    ("chunk", 2, 28, 4, 70, [600, 333], [70, 65], "causal", 8.0, False),
    ("chunk_docs", 2, 8, 1, 130, [400, 130], None, "docs", 0.0, False),
    ("chunk_docs_prefix", 1, 6, 2, 190, [555], None, "docs_prefix", 20.0, True),
    ("chunk_window", 1, 3, 1, 300, [300], None, "window", 0.0, False),
    ("chunk_both_ways", 1, 4, 2, 90, [90], None, "both_ways", 0.0, True),
    ("chunk_holes", 2, 8, 8, 100, [260, 100], [100, 30], "holes", 0.0, False),
    ("split_rows", 1, 2, 1, 40, [3000], None, "causal", 0.0, False),
    ("split_docs", 1, 2, 2, 33, [2500], None, "docs", 0.0, True),
    ("beyond_the_capacity", 1, 2, 1, 30, [100], None, "causal", 0.0, False),     # capacity 96: the last rows are not there
]


def inputs(case, seed=3):
    name, B, Hq, H, T, lens, new, kind, cap, slopes = case
    rows = 96 if name == "beyond_the_capacity" else (max(max(lens), 1) + 7) // 8 * 8
    g = torch.Generator().manual_seed(seed)
    q = (torch.randn(B, T, Hq, 128, generator=g) * (3.0 if cap else 1.0)).to(torch.bfloat16)
    K, V = (torch.randn(B, H, rows, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    nl = [T] * B if new is None else new
    first, end = ranges(kind, B, T, lens, nl, seed)
    sl = torch.exp2(-torch.arange(1, Hq + 1).float() * 6 / Hq) if slopes else None
    return q, K, V, nl, first, end, sl


def dev(x, dtype=torch.int32):
    return None if x is None else (torch.from_numpy(x).cuda() if isinstance(x, np.ndarray) else x.cuda() if isinstance(x, torch.Tensor) else torch.tensor(x, dtype=dtype, device="cuda"))


def close(case, geom, q, K, V, nl, first, end, slopes, out, lse, seen_rows=None):
    """Scores: 128 products added in fp32 and five roundings of the cap and the bias, 140 * 2^-24 of their terms' sizes and 2^-21 of the cap (tanh by
    1 - 2 / (e^2x + 1), the exponential and the reciprocal good to 2^-22).  Weights: twice that, 2^-20, 2^-22 of s - max; in the product with V
    2^-8 where they are bf16 (more than 16 rows of a group), 2^-16 otherwise.  The output is rounded once, 2^-8."""
    name, B, Hq, H, T, lens, _, kind, cap, _ = case
    G, scale = Hq // H, geom.scale
    a, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    qf, Kf, Vf = (x.double().numpy() for x in (q, K, V))
    few = T * G <= 16
    for b in range(B):
        rows = min(lens[b], K.shape[2])
        for i in range(nl[b]):
            p = lens[b] - nl[b] + i
            lo, hi = (0, p + 1) if first is None else (int(first[b, i]), int(end[b, i]))
            hi = min(hi, rows)
            for h in range(Hq):
                s1 = 0.0 if slopes is None else float(slopes[h])
                want, wl = o.prompt_attn(qf[b, i, h], Kf[b, h // G, :rows], Vf[b, h // G, :rows], p, lo, hi, scale, cap, s1)
                what = (name, b, i, h)
                if hi <= max(lo, 0):
                    assert (a[b, i, h] == 0).all() and l[b, i, h] == -math.inf, what
                    continue
                j = np.arange(max(lo, 0), hi)
                k, v = Kf[b, h // G, j], Vf[b, h // G, j]
                s = scale * (k @ qf[b, i, h])
                size = scale * (np.abs(k) @ np.abs(qf[b, i, h])) + s1 * np.abs(p - j)
                if cap:
                    s = cap * np.tanh(s / cap)
                s = s - s1 * np.abs(p - j)
                ds = 140 * 2.0 ** -24 * size.max() + 2.0 ** -21 * cap
                w = np.exp(s - s.max())
                w /= w.sum()
                rel = 2 * ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(s - s.max()) + (2.0 ** -16 if few else 2.0 ** -8)
                assert abs(l[b, i, h] - wl) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wl), (what, l[b, i, h], wl)
                err = 2.0 ** -8 * np.abs(want) + (rel * w) @ np.abs(v)
                assert (np.abs(a[b, i, h] - want) <= err).all(), (what, np.abs(a[b, i, h] - want).max())
    for b in range(B):                                                           # entries that are none are left alone
        assert (a[b, nl[b]:] == 9).all() and (l[b, nl[b]:] == 9).all(), name


@gpu
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_attn(rk, case):
    name, B, Hq, H, T, lens, new, kind, cap, _ = case
    say("prompt", name)
    q, K, V, nl, first, end, slopes = inputs(case)
    geom = rk.Geom(B, Hq, H, 128, float(np.float32(1 / np.sqrt(128))))
    # what no sequence has is NaN, and K and V are pieces of something larger
    Kn, Vn = K.clone(), V.clone()
    for b in range(B):
        Kn[b, :, lens[b]:] = math.nan
        Vn[b, :, lens[b]:] = math.nan
    wide = torch.full((B, H, 2, K.shape[2] + 8, 128), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:, :, 0, :K.shape[2]], wide[:, :, 1, :K.shape[2]] = Kn.cuda(), Vn.cuda()
    Kd, Vd = wide[:, :, 0, :K.shape[2]], wide[:, :, 1, :K.shape[2]]
    qw = torch.zeros(B, T, Hq + 3, 128, dtype=torch.bfloat16, device="cuda")
    qw[:, :, 1:1 + Hq] = q.cuda()
    out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
    ws = rk.PromptWorkspace(geom, T, K.shape[2])
    args = dict(new_lens=None if new is None else dev(nl), first=dev(first), end=dev(end), cap=cap, slopes=dev(slopes), workspace=ws)
    rk.rk_prompt_attn(geom, qw[:, :, 1:1 + Hq], Kd, Vd, dev(lens), K.shape[2], out, lse=lse, **args)
    torch.cuda.synchronize()
    close(case, geom, q, K, V, nl, first, end, slopes, out, lse)
    again = torch.full_like(out, 9.0)
    rk.rk_prompt_attn(geom, q.cuda(), Kd, Vd, dev(lens), K.shape[2], again, **args)
    assert torch.equal(out, again)


@gpu
@pytest.mark.parametrize("case", [c for c in CASES if c[0] in ("drafted", "drafted_holes", "drafted_16", "whole_prompt", "chunk_docs", "chunk_docs_prefix", "split_docs", "chunk_window")],
                         ids=lambda c: c[0])
def test_rows_that_a_token_does_not_see_have_no_part(rk, case):
    """Infinities and NaN planted in K and V: tokens that do not see them get what they get without; tokens that do see one get what comes of it."""
    name, B, Hq, H, T, lens, new, kind, cap, _ = case
    say("planted", name)
    q, K, V, nl, first, end, slopes = inputs(case)
    geom = rk.Geom(B, Hq, H, 128, float(np.float32(1 / np.sqrt(128))))
    r = np.random.default_rng(1)
    K2, V2 = K.clone(), V.clone()
    planted = []
    for b in range(B):
        for j in sorted(set(r.integers(0, lens[b], 3).tolist()) | {lens[b] - 2}):
            g, d, v = int(r.integers(H)), int(r.integers(128)), [math.inf, -math.inf, math.nan][int(r.integers(3))]
            V2[b, g, j, d] = v
            planted.append((b, g, j, d, v))
        K2[b, 0, lens[b] - 1, 5] = math.nan                                       # the last row: seen by the last token, and through prefixes
    outs = []
    for k, v in ((K, V), (K2, V2)):
        out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
        rk.rk_prompt_attn(geom, q.cuda(), k.cuda(), v.cuda(), dev(lens), K.shape[2], out, lse=lse, new_lens=None if new is None else dev(nl), first=dev(first),
                          end=dev(end), cap=cap, slopes=dev(slopes), workspace=rk.PromptWorkspace(geom, T, K.shape[2]))
        outs.append((out.double().cpu().numpy(), lse.double().cpu().numpy()))
    (a, la), (c, lc) = outs
    G = Hq // H
    for b in range(B):
        for i in range(nl[b]):
            p = lens[b] - nl[b] + i
            lo, hi = (0, p + 1) if first is None else (max(int(first[b, i]), 0), min(int(end[b, i]), lens[b]))
            for g in range(H):
                hs = slice(g * G, (g + 1) * G)
                if g == 0 and lo <= lens[b] - 1 < hi:
                    assert np.isnan(c[b, i, hs]).all() and np.isnan(lc[b, i, hs]).all(), (name, b, i)
                    continue
                assert (la[b, i, hs] == lc[b, i, hs]).all(), (name, b, i, g)
                want = a[b, i, hs].copy()
                for bb, gg, j, d, v in planted:
                    if bb == b and gg == g and lo <= j < hi:
                        want[:, d] += v
                if T * G <= 16:                                                   # (weights in two parts: an infinity may come out as NaN)
                    assert (np.isfinite(c[b, i, hs]) == np.isfinite(want)).all(), (name, b, i, g)
                    want = np.where(np.isfinite(want), want, c[b, i, hs])
                np.testing.assert_array_equal(c[b, i, hs], want, err_msg=str((name, b, i, g)))


@gpu
def test_predicate_max_len_and_two_streams(rk):
    B, Hq, H, T = 2, 8, 2, 60
    geom = rk.Geom(B, Hq, H, 128, 0.1)
    g = torch.Generator().manual_seed(0)
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16).cuda()
    K, V = (torch.randn(B, H, 512, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    sl = dev([500, 400])
    # with max_len, rows from there on are not looked at: as if the ranges ended there
    out, cut, ws = torch.zeros_like(q), torch.zeros_like(q), rk.PromptWorkspace(geom, T, 512)
    end = (sl[:, None] - T + 1 + torch.arange(T, device="cuda")).clamp(max=130).int()
    rk.rk_prompt_attn(geom, q, K, V, sl, 130, out, workspace=ws)
    rk.rk_prompt_attn(geom, q, K, V, sl, 512, cut, end=end, workspace=ws)
    assert (out.double() - cut.double()).abs().max() <= 2.0 ** -6 * out.double().abs().max()      # (splits of their own)
    pred = dev([0, 1])
    only = torch.full_like(q, 3.0)
    rk.rk_prompt_attn(geom, q, K, V, sl, 512, only, pred=pred, pred_val=1, workspace=ws)
    full = torch.zeros_like(q)
    rk.rk_prompt_attn(geom, q, K, V, sl, 512, full, workspace=ws)
    assert (only[0] == 3).all() and torch.equal(only[1], full[1])
    # two calls at once, each with its own scratch
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], []
    for s in streams:
        with torch.cuda.stream(s):
            x, w = torch.zeros_like(q), rk.PromptWorkspace(geom, T, 512)
            for _ in range(10):
                rk.rk_prompt_attn(geom, q, K, V, sl, 512, x, workspace=w)
            got.append(x)
    torch.cuda.synchronize()
    assert torch.equal(got[0], full) and torch.equal(got[1], full)


@gpu
def test_a_long_split_step_and_its_parts_agree(rk):
    """One token over 40000 rows, many splits, a window of one row at both ends; and captured."""
    geom = rk.Geom(1, 8, 2, 128, 0.1)
    g = torch.Generator().manual_seed(6)
    n = 40000
    q = torch.randn(1, 1, 8, 128, generator=g).to(torch.bfloat16)
    K, V = (torch.randn(1, 2, n, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    case = ("long", 1, 8, 2, 1, [n], None, "causal", 0.0, False)
    ws = rk.PromptWorkspace(geom, 1, n)
    qd, Kd, Vd, sl = q.cuda(), K.cuda(), V.cuda(), dev([n])
    out, lse = torch.zeros_like(qd), torch.zeros(1, 1, 8, device="cuda")
    rk.rk_prompt_attn(geom, qd, Kd, Vd, sl, n, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    close(case, geom, q, K, V, [1], None, None, None, out, lse)
    for j in (0, n - 1, 20001):
        one = torch.zeros_like(qd)
        rk.rk_prompt_attn(geom, qd, Kd, Vd, sl, n, one, first=dev([[j]]), end=dev([[j + 1]]), workspace=ws)
        assert torch.equal(one[0, 0], Vd[0, :, j].repeat_interleave(4, dim=0)), j
    graph, held, hl = torch.cuda.CUDAGraph(), torch.zeros_like(qd), torch.zeros_like(lse)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rk.rk_prompt_attn(geom, qd, Kd, Vd, sl, n, held, lse=hl, workspace=ws)
    for m in (n, 777, 1, 0, 12345):
        sl.fill_(m)
        graph.replay()
        rk.rk_prompt_attn(geom, qd, Kd, Vd, sl, n, out, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(held, out) and torch.equal(hl, lse), m


@gpu
def test_chunks_are_the_whole_prompt(rk):
    """A prompt in chunks through append and attention gives what it gives in one piece (and the last token alone, as a decode step)."""
    B, Hq, H, n = 1, 8, 2, 300
    geom = rk.Geom(B, Hq, H, 128, 0.1)
    g = torch.Generator().manual_seed(2)
    w = torch.randn(B, n, Hq + 2 * H, 128, generator=g).to(torch.bfloat16).cuda()
    q, k, v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
    rope, ws = rk.Rope(rk.rope_table(n, 128)), rk.PromptWorkspace(geom, n, 304)

    def run(pieces):
        K, V = (torch.zeros(B, H, 304, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        outs, at = [], 0
        for t in pieces:
            qo, out = (torch.zeros(B, t, Hq, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            sl = dev([at + t])
            rk.rk_rope_append(geom, q[:, at:at + t], k[:, at:at + t], v[:, at:at + t], rope, K, V, sl, qo)
            rk.rk_prompt_attn(geom, qo, K, V, sl, 304, out, workspace=ws)
            outs.append(out)
            at += t
        return torch.cat(outs, dim=1).double(), K, V
    whole, K, V = run([n])
    for pieces in ([128, 128, 44], [1, 2, 290, 3, 4], [299, 1]):
        x, K2, V2 = run(pieces)
        assert torch.equal(K, K2) and torch.equal(V, V2)
        # both are within 2^-8 of the weights' rounding and half a step of the output's: four times 2^-8 of the values' size (at most about 4 sigma of V)
        assert (x - whole).abs().max() <= 4 * 2.0 ** -8 * float(v.double().abs().max())
