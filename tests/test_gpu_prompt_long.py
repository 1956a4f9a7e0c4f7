"""rk_prompt_attn where it has so many rows that a wavefront takes 64 of them: against oracle/new_tokens.py, at rows drawn from all of them."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import new_tokens as o
from test_gpu_prompt_attn import close, ranges

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))
B, Hq, H, T, CAP = 8, 32, 16, 512, 704          # 128 (sequence, KV head) pairs of 1024 rows: 512 workgroups of 256


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def i32(x):
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def check(q, K, V, lens, new, first, end, scale, out, lse, seed, n=400, what=""):
    """Tolerances as in test_gpu_prompt_attn.close, for more than 16 rows of a group."""
    r = np.random.default_rng(seed)
    a, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    G = Hq // H
    for x in range(n):
        b = x % B
        if new[b] == 0:
            continue
        i, h = int(r.integers(0, new[b])) if x >= 2 * B else (0 if x < B else new[b] - 1), int(r.integers(0, Hq))
        p = lens[b] - new[b] + i
        lo, hi = (0, p + 1) if first is None else (int(first[b, i]), int(end[b, i]))
        hi = min(hi, lens[b])
        kf, vf, qf = K[b, h // G, :lens[b]].double().numpy(), V[b, h // G, :lens[b]].double().numpy(), q[b, i, h].double().numpy()
        want, wl = o.prompt_attn(qf, kf, vf, p, lo, hi, scale)
        at = (what, b, i, h)
        if hi <= max(lo, 0):
            assert (a[b, i, h] == 0).all() and l[b, i, h] == -math.inf, at
            continue
        k, v = kf[max(lo, 0):hi], vf[max(lo, 0):hi]
        s = scale * (k @ qf)
        ds = 140 * 2.0 ** -24 * abs(scale) * float((np.abs(k) @ np.abs(qf)).max())
        w = np.exp(s - s.max())
        w /= w.sum()
        rel = 2 * ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(s - s.max()) + 2.0 ** -8
        assert abs(l[b, i, h] - wl) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wl), (at, l[b, i, h], wl)
        assert (np.abs(a[b, i, h] - want) <= 2.0 ** -8 * np.abs(want) + (rel * w) @ np.abs(v)).all(), at
    for b in range(B):
        assert (a[b, new[b]:] == 9).all() and (l[b, new[b]:] == 9).all(), what


@pytest.mark.parametrize("kind,scale,gain", [("causal", SCALE, 1.0), ("causal", -SCALE, 6.0), ("docs", SCALE, 1.0), ("docs_prefix", SCALE, 3.0), ("window", SCALE, 1.0),
                                             ("both_ways", SCALE, 1.0), ("holes", SCALE, 1.0)])
def test_attn(rk, kind, scale, gain):
    print("long", kind, scale, file=sys.stderr, flush=True)
    geom = rk.Geom(B, Hq, H, 128, scale)
    g = torch.Generator().manual_seed(31)
    lens, new = [700, 512, 1, 9, 513, 640, 699, 257], [512, 512, 1, 0, 512, 33, 511, 257]
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16)
    # (keys that grow along the rows: the maximum moves again and again)
    K = (torch.randn(B, H, CAP, 128, generator=g) * torch.linspace(1, gain, CAP)[:, None]).to(torch.bfloat16)
    V = torch.randn(B, H, CAP, 128, generator=g).to(torch.bfloat16)
    for b, m in enumerate(lens):
        K[b, :, m:], V[b, :, m:] = math.nan, math.nan
    first, end = ranges(kind, B, T, lens, new, 5)
    out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
    ws = rk.PromptWorkspace(geom, T, CAP)
    rk.rk_prompt_attn(geom, q.cuda(), K.cuda(), V.cuda(), i32(lens), CAP, out, new_lens=i32(new), first=None if first is None else i32(first),
                      end=None if end is None else i32(end), lse=lse, workspace=ws)
    torch.cuda.synchronize()
    check(q, K, V, lens, new, first, end, scale, out, lse, 7, what=kind)


def test_rows_that_a_token_does_not_see_have_no_part(rk):
    """Infinities and NaN in V: a token that sees one gets it, the others of its tile do not; NaN among keys that nothing sees."""
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(32)
    lens, new = [700, 512, 600, 550, 513, 640, 699, 257], [512, 512, 512, 300, 512, 33, 511, 257]
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16)
    K, V = (torch.randn(B, H, CAP, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    first, end = ranges("window", B, T, lens, new, 5)
    bad = [(b, h, m - 40, d) for b, m in enumerate(lens) for h, d in ((0, 5), (H - 1, 127))]
    clean = V.clone()
    for x, (b, h, j, d) in enumerate(bad):
        V[b, h, j, d] = (math.inf, -math.inf, math.nan)[x % 3]
        clean[b, h, j, d] = 0
    hidden = K.clone()
    for b, m in enumerate(lens):
        seen = np.zeros(CAP, bool)
        for i in range(new[b]):
            seen[max(first[b, i], 0):min(end[b, i], m)] = True
        hidden[b][:, torch.from_numpy(~seen)] = math.nan
    got = []
    for k, v in ((K, clean), (hidden, V)):
        out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
        rk.rk_prompt_attn(geom, q.cuda(), k.cuda(), v.cuda(), i32(lens), CAP, out, new_lens=i32(new), first=i32(first), end=i32(end), lse=lse,
                          workspace=rk.PromptWorkspace(geom, T, CAP))
        torch.cuda.synchronize()
        got.append((out.cpu(), lse.cpu()))
    assert torch.equal(got[0][1], got[1][1])
    expect = got[0][0].clone()
    touched = torch.zeros(expect.shape, dtype=torch.bool)
    G = Hq // H
    for b, h, j, d in bad:
        for i in range(new[b]):
            if max(first[b, i], 0) <= j < min(end[b, i], lens[b]):
                touched[b, i, h * G:(h + 1) * G, d] = True
    assert touched.any() and not got[1][0][touched].isfinite().any()
    assert torch.equal(got[1][0][~touched], expect[~touched])


def test_predicate_and_captured(rk):
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator(device="cuda").manual_seed(33)
    q = torch.randn(B, T, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    K, V = (torch.randn(B, H, CAP, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    sl, pred = i32([700, 512, 600, 550, 513, 640, 699, 512]), i32([1, 0] * 4)
    held, eager = (torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    call = lambda o_: rk.rk_prompt_attn(geom, q, K, V, sl, CAP, o_, pred=pred, pred_val=1)  # noqa: E731  (nothing is split: no workspace)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(held)
    for lens in ([700, 512, 600, 550, 513, 640, 699, 512], [512] * 8, [3, 700, 0, 1, 699, 2, 511, 600]):
        sl.copy_(i32(lens))
        held.fill_(9), eager.fill_(9)
        graph.replay()
        call(eager)
        torch.cuda.synchronize()
        assert torch.equal(held, eager) and (held[1::2] == 9).all()


@pytest.mark.parametrize("kind,cap,slopes", [("causal", 0.0, False), ("causal", 5.0, True), ("docs", 0.0, True), ("holes", 4.0, False)])
@pytest.mark.parametrize("n_b,hq,h,t,rows", [(16, 16, 8, 3, 500), (20, 28, 4, 1, 512), (17, 8, 8, 16, 640), (70, 8, 4, 2, 700)])
def test_few_tokens_of_many_heads(rk, kind, cap, slopes, n_b, hq, h, t, rows):
    """A workgroup alone with all rows of a (sequence, KV head), of ragged sequences; what none of them has is NaN."""
    geom = rk.Geom(n_b, hq, h, 128, SCALE)
    g = torch.Generator().manual_seed(n_b)
    lens = [1 + (173 * i) % rows for i in range(n_b)]
    new = [min(m, t) if i % 4 else min(m, 1) for i, m in enumerate(lens)]
    q = (torch.randn(n_b, t, hq, 128, generator=g) * 2).to(torch.bfloat16)
    K, V = (torch.randn(n_b, h, rows, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    for b, m in enumerate(lens):
        K[b, :, m:], V[b, :, m:] = math.nan, math.nan
    first, end = ranges(kind, n_b, t, lens, new, 9)
    sl = torch.exp2(-torch.arange(1, hq + 1).float() * 6 / hq) if slopes else None
    out, lse = torch.full((n_b, t, hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((n_b, t, hq), 9.0, device="cuda")
    rk.rk_prompt_attn(geom, q.cuda(), K.cuda(), V.cuda(), i32(lens), rows, out, new_lens=i32(new), first=None if first is None else i32(first),
                      end=None if end is None else i32(end), cap=cap, slopes=None if sl is None else sl.cuda(), lse=lse, workspace=rk.PromptWorkspace(geom, t, rows))
    torch.cuda.synchronize()
    close(("alone", n_b, hq, h, t, lens, new, kind, cap, slopes), geom, q, K, V, new, first, end, sl, out, lse)
