"""rk_full_attn_q8, rk_gather_small_kv_q8: refusals (no GPU needed), and against oracle/new_tokens.py."""
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
    from paper_2411_05787_amd.binding import _Geom, _Kv, _Kv8
    g, f = _Geom(2, 32, 8, 128, 0.1), 0x10000
    wsb = rk.workspace_bytes(rk.Geom(2, 32, 8, 128, 0.1), 64, 1)
    c8 = lambda k=f, block=32, fmt=0: _Kv8(k, f, f, f, f, f, 8 * 64 * 128, 64 * 128, 64, block, fmt)  # noqa: E731

    def attn(geom=g, q=f, c=c8(), sl=f, max_len=64, out=f, w=None, ws_=0, ws=0x100000, nb=wsb):
        return rk.lib.rk_full_attn_q8(C.byref(geom), q, None if c is None else C.byref(c), sl, max_len, out, w, ws_, None, None, 0, ws, nb, None)

    assert attn(geom=_Geom(2, 72, 8, 128, 0.1)) == -2 and attn(geom=_Geom(2, 32, 8, 64, 0.1)) == -2
    assert attn(q=None) == -1 and attn(out=None) == -1 and attn(sl=None) == -1 and attn(max_len=0) == -1 and attn(c=None) == -1
    assert attn(q=f + 8) == -1 and attn(out=f + 1) == -1 and attn(c=c8(k=f + 8)) == -1
    assert attn(c=c8(block=24)) == -2 and attn(c=c8(fmt=7)) == -2
    assert attn(w=f, ws_=60) == -1 and attn(w=f + 2, ws_=64) == -1
    assert attn(ws=None) == -3 and attn(ws=0x100010) == -3 and attn(nb=1024) == -3
    small = _Kv(f, f, 8 * 16 * 128, 16 * 128, 16)
    gather = lambda c=c8(), idx=f, k=16, s=small, sl=f: rk.lib.rk_gather_small_kv_q8(C.byref(g), C.byref(c), idx, k, s, sl, None, None, 0, None)  # noqa: E731
    assert gather(idx=None) == -1 and gather(k=0) == -1 and gather(sl=None) == -1 and gather(k=17) == -1
    assert gather(s=_Kv(f, None, 0, 0, 16)) == -1 and gather(c=c8(fmt=3)) == -2


def test_binding_refuses(rk):
    g = rk.Geom(1, 4, 2, 128, 0.1)
    with pytest.raises(ValueError):
        rk.rk_full_attn_q8(g, torch.zeros(1, 4, 128, dtype=torch.bfloat16), None, torch.zeros(1, dtype=torch.int32), 8, None)


def make(rk, seed, B, H, cap, block, fmt, lens, gain=1.0, powers=True, strided=False):
    """A cache of random bytes and scales; whatever no sequence has is NaN."""
    g = torch.Generator().manual_seed(seed)
    dtype = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    geom_b = B
    t = {}
    for n in "kv":
        if fmt == "e4m3":
            x = torch.randn(geom_b, H, cap, 128, generator=g).mul(100).clamp(-448, 448).to(dtype).view(torch.uint8)
        else:
            x = torch.randint(-127, 128, (geom_b, H, cap, 128), generator=g).to(torch.int8).view(torch.uint8)
        e = torch.randint(-2, 3, (geom_b, H, cap // block), generator=g).float()
        s = (torch.exp2(e) if powers else torch.exp(0.7 * torch.randn(geom_b, H, cap // block, generator=g))) * (2.0 ** -6) * (gain if n == "k" else 1.0)
        tail = torch.randn(geom_b, H, block, 128, generator=g).to(torch.bfloat16)
        for b, m in enumerate(lens):
            m = min(max(m, 0), cap)
            full = m // block
            x[b, :, full * block:] = 0x7f                                         # NaN in e4m3, 127 in int8
            s[b, :, full:] = math.nan
            tail[b, :, m - full * block:] = math.nan
        t[n + "8"], t[n + "_scale"], t[n + "_tail"] = x, s, tail
    dev = {}
    for n in "kv":
        x = t[n + "8"].cuda()
        if strided:                                                              # [H, B, ..] with room between
            wide = torch.full((H, B, cap + 16, 128), 0x7f, dtype=torch.uint8, device="cuda")
            wide[:, :, :cap] = x.transpose(0, 1)
            x = wide[:, :, :cap].transpose(0, 1)
        dev[n] = x.view(dtype)
    values = {}
    for n in "kv":
        values[n] = t[n + "8"].view(dtype).double().numpy(), t[n + "_scale"].double().numpy(), t[n + "_tail"].double().numpy()
    geom = None

    def rows(n, b, h, m):
        x, s, tail = values[n]
        full = m // block
        return np.concatenate([x[b, h, :full * block] * np.repeat(s[b, h, :full], block)[:, None], tail[b, h, :m - full * block]])
    return lambda geom: rk.Kv8(geom, dev["k"], dev["v"], t["k_scale"].cuda(), t["v_scale"].cuda(), t["k_tail"].cuda(), t["v_tail"].cuda()), rows


def check(q, rows, scale, b, G, h, m, out, lse, w, what, rounded=False):
    """Scores: 128 products added in fp32 and two more roundings, 131 * 2^-24 of sum |q k|; a weight's exponent is off by twice that and by the
    rounding of s - max times log2 e (2^-22 relative), the exponential by 2^-22; P is kept to 2^-17, sums to 2^-20; the output is rounded once (2^-8)."""
    k, v = rows("k", b, h // G, m), rows("v", b, h // G, m)
    want, p, wl = o.attn8(gen.bf16_bits(q)[b, h], k, v, scale)
    if m == 0:
        assert (out[b, h] == 0).all() and lse[b, h] == -math.inf, what
        return
    qa = np.abs(o.bf16_bits_to_f64(gen.bf16_bits(q)[b, h]))
    s = scale * (k @ o.bf16_bits_to_f64(gen.bf16_bits(q)[b, h]))
    ds = 131 * 2.0 ** -24 * scale * float((np.abs(k) @ qa).max())
    rel = 2 * ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(s - s.max())
    assert abs(lse[b, h] - wl) <= ds + 2.0 ** -20 + 2.0 ** -23 * abs(wl), (what, lse[b, h], wl)
    if w is not None:
        assert (np.abs(w[b, h, :m] - p) <= (rel + 2.0 ** -22 * abs(wl)) * p + 1e-38).all(), what
    err = 2.0 ** -8 * np.abs(want) + ((rel + 2.0 ** -16) * p) @ np.abs(v)
    assert (np.abs(out[b, h] - want) <= err).all(), (what, np.abs(out[b, h] - want).max())


CASES = [
    # name, B, Hq, H, block, format, lens, cap
    ("g4", 1, 32, 8, 32, "e4m3", [777], 800),
    ("g7_int8", 1, 28, 4, 64, "int8", [1001], 1024),
    ("g1_block16", 2, 2, 2, 16, "e4m3", [47, 48], 64),
    ("g8_block128", 1, 8, 1, 128, "int8", [1155], 1280),
    ("g3", 1, 9, 3, 16, "int8", [33], 48),
    ("g5_tail_alone", 2, 5, 1, 128, "e4m3", [127, 1], 128),
    ("empty_and_one", 4, 8, 2, 32, "e4m3", [0, 1, 32, 31], 64),
    ("ragged", 6, 8, 2, 32, "int8", [3000, 5, 0, 1500, 129, 2999], 3008),
    ("ragged_even", 65, 4, 1, 16, "e4m3", [(i * 37) % 300 for i in range(65)], 304),
    ("long", 1, 16, 4, 64, "e4m3", [9001], 9024),
    ("beyond_the_capacity", 2, 4, 2, 32, "e4m3", [70, 64], 64),
]


@gpu
@pytest.mark.parametrize("powers", [True, False], ids=["powers", "any_scale"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_attn(rk, case, powers):
    name, B, Hq, H, block, fmt, lens, cap = case
    say("q8 attn", name, powers)
    scale = float(np.float32(1 / np.sqrt(128)))
    geom = rk.Geom(B, Hq, H, 128, scale)
    cache, rows = make(rk, 7, B, H, cap, block, fmt, lens, powers=powers, strided=not powers)
    cache = cache(geom)
    q = torch.randn(B, Hq, 128, generator=torch.Generator().manual_seed(8)).to(torch.bfloat16)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = rk.Workspace(geom, cap, 1)
    width = cap + (0 if powers else 3)                                           # rows that do and do not start on 16 bytes
    out, lse = torch.full((B, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq), 9.0, device="cuda")
    w = torch.full((B, Hq, width), -7.0, device="cuda")
    rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, cap, out, weights=w, lse=lse, workspace=ws)
    out2, lse2 = torch.zeros_like(out), torch.zeros_like(lse)
    rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, cap, out2, lse=lse2, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, out2)                                                # with weights or without
    a, l, wn = out.double().cpu().numpy(), lse.double().cpu().numpy(), w.double().cpu().numpy()
    for b, m in enumerate(lens):
        m = min(m, cap)
        for h in range(Hq):
            check(q, rows, scale, b, Hq // H, h, m, a, l, wn, "%s %d %d" % (name, b, h))
        assert (wn[b, :, m:] == -7).all()


@gpu
def test_max_len_predicate_and_large_scores(rk):
    B, Hq, H, cap, block = 3, 8, 2, 512, 32
    scale = 0.25
    geom = rk.Geom(B, Hq, H, 128, scale)
    lens = [512, 300, 431]
    cache, rows = make(rk, 3, B, H, cap, block, "e4m3", lens, gain=4.0)          # scores of some hundreds
    cache = cache(geom)
    q = torch.randn(B, Hq, 128, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    ws = rk.Workspace(geom, cap, 1)
    for max_len in (512, 301, 7):
        out, lse = torch.full((B, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq), 9.0, device="cuda")
        pred = torch.tensor([1, 1, 0], dtype=torch.int32, device="cuda")
        rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, max_len, out, lse=lse, pred=pred, pred_val=1, workspace=ws)
        torch.cuda.synchronize()
        assert (out[2] == 9).all() and (lse[2] == 9).all()
        for b in (0, 1):
            for h in range(Hq):
                cut = lambda n, bb, hh, m, b=b: rows(n, bb, hh, lens[b])[:m]     # rows beyond max_len exist, in their blocks  # noqa: E731
                check(q, cut, scale, b, Hq // H, h, min(lens[b], max_len), out.double().cpu().numpy(), lse.double().cpu().numpy(), None, (max_len, b, h))


@gpu
def test_a_block_that_held_a_nan_is_nan(rk):
    geom = rk.Geom(2, 4, 2, 128, 0.1)
    cache = rk.Kv8.empty(geom, 64, 32, torch.int8)
    x = torch.randn(2, 64, 2, 128, device="cuda").to(torch.bfloat16)
    x[0, 40, 1, 3] = float("inf")
    sl = torch.tensor([64, 64], dtype=torch.int32, device="cuda")
    rk.rk_rope_append_q8(geom, None, x, x, None, cache, sl, None)
    out, lse, w = torch.zeros(2, 4, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 4, device="cuda"), torch.zeros(2, 4, 64, device="cuda")
    q = torch.randn(2, 4, 128, device="cuda").to(torch.bfloat16)
    rk.rk_full_attn_q8(geom, q, cache, sl, 64, out, weights=w, lse=lse, workspace=rk.Workspace(geom, 64, 1))
    assert out[0, 2:].isnan().all() and lse[0, 2:].isnan().all() and w[0, 2:].isnan().all()
    assert out[0, :2].isfinite().all() and out[1].isfinite().all() and w[1].isfinite().all()


@gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_gather(rk, fmt):
    B, H, cap, block, k = 3, 2, 256, 32, 70
    lens = [256, 77, 0]
    geom = rk.Geom(B, 4, H, 128, 0.1)
    cache, rows = make(rk, 11, B, H, cap, block, fmt, lens, strided=True)
    cache = cache(geom)
    r = np.random.default_rng(0)
    idx = r.integers(-1, cap + 40, (B, H, k)).astype(np.int32)
    idx[0, 0, :3], idx[1, 0, :4] = [255, 0, 255], [76, 63, 64, 77]               # the last row, the first, one twice; the tail, the block before it, none
    wide = torch.full((B, H, 2, k + 4, 128), 5.0, dtype=torch.bfloat16, device="cuda")
    sK, sV = wide[:, :, 0], wide[:, :, 1]
    ts = torch.full((B,), -1, dtype=torch.int32, device="cuda")
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    rk.rk_gather_small_kv_q8(geom, cache, torch.from_numpy(idx).cuda(), k, sK, sV, sl, tail_start=ts)
    torch.cuda.synchronize()
    assert ts.tolist() == lens
    for n, s in (("k", sK), ("v", sV)):
        got = s.double().cpu().numpy()
        assert (got[:, :, k:] == 5).all()
        for b in range(B):
            for h in range(H):
                have = rows(n, b, h, lens[b])
                for i in range(k):
                    j = idx[b, h, i]
                    assert (got[b, h, i] == (have[j] if 0 <= j < lens[b] else 5.0)).all(), (n, b, h, i, j)
    pred = torch.tensor([0, 1, 1], dtype=torch.int32, device="cuda")
    wide.fill_(5.0)
    rk.rk_gather_small_kv_q8(geom, cache, torch.from_numpy(idx).cuda(), k, sK, sV, sl, pred=pred, pred_val=1)
    assert (wide[0] == 5).all() and not (wide[1] == 5).all()


@gpu
def test_captured_and_on_another_stream(rk):
    """A step (append, attention with weights, selection, gather) captured once and replayed over growing caches is the eager one."""
    B, Hq, H, cap, block, k = 2, 8, 2, 256, 32, 24
    geom = rk.Geom(B, Hq, H, 128, 0.09)
    g = torch.Generator(device="cuda").manual_seed(4)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        rope = rk.Rope(rk.rope_table(cap, 64))

        def state():
            s = dict(cache=rk.Kv8.empty(geom, cap, block), sl=torch.tensor([90, 31], dtype=torch.int32, device="cuda"), ws=rk.Workspace(geom, cap, k),
                     out=torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda"), w=torch.zeros(B, Hq, cap, device="cuda"),
                     qo=torch.zeros(B, 1, Hq, 128, dtype=torch.bfloat16, device="cuda"), idx=torch.zeros(B, H, k, dtype=torch.int32, device="cuda"),
                     small=torch.zeros(2, B, H, k, 128, dtype=torch.bfloat16, device="cuda"))
            x = torch.randn(B, 90, 2 * H, 128, generator=torch.Generator(device="cuda").manual_seed(9), device="cuda").to(torch.bfloat16)
            rk.rk_rope_append_q8(geom, None, x[:, :, :H], x[:, :, H:], rope, s["cache"], s["sl"], None, new_lens=s["sl"])
            return s

        new = torch.zeros(B, 1, Hq + 2 * H, 128, dtype=torch.bfloat16, device="cuda")

        def step(s):
            s["sl"] += 1
            rk.rk_rope_append_q8(geom, new[:, :, :Hq], new[:, :, Hq:Hq + H], new[:, :, Hq + H:], rope, s["cache"], s["sl"], s["qo"])
            rk.rk_full_attn_q8(geom, s["qo"].view(B, Hq, 128), s["cache"], s["sl"], cap, s["out"], weights=s["w"], workspace=s["ws"])
            rk.rk_topk_select(geom, s["w"], s["sl"], cap, k, 7, s["idx"], workspace=s["ws"])
            rk.rk_gather_small_kv_q8(geom, s["cache"], s["idx"], k, s["small"][0], s["small"][1], s["sl"])

        eager, held = state(), state()
        step(state())                                                            # (first launches outside the capture)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            step(held)
        for i in range(40):
            new.copy_(torch.randn(new.shape, generator=g, device="cuda"))
            graph.replay()
            step(eager)
            torch.cuda.synchronize()
            for n in ("out", "qo", "idx", "small", "sl"):
                assert torch.equal(held[n], eager[n]), (i, n)
            for n in ("k", "v"):
                assert torch.equal(getattr(held["cache"], n).view(torch.uint8), getattr(eager["cache"], n).view(torch.uint8))
        assert eager["sl"].tolist() == [130, 71]
