"""rk_paged_attn with 64 rows to a wavefront, which calls take that make two rounds of workgroups of 256 rows (512 and more (sequence, KV head, 256 rows)),
without cap or bias: pages that are none, pages of every size, pools in parts of something larger, ranges, rows behind one register of page numbers,
infinities and NaN.  Against oracle/paged.py."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as o
from test_gpu_paged_attn import Inputs, rk, say  # noqa: F401

pytestmark = pytest.mark.gpu


def some(n, most, seed):
    return np.random.default_rng(seed).integers(1, most + 1, n).tolist()


CASES = {
    "missing": dict(B=64, Hq=8, H=8, T=20, lens=some(64, 300, 1), new=[min(20, n) for n in some(64, 300, 1)], page=16, missing=3),
    "missing_32": dict(B=32, Hq=32, H=16, T=12, lens=some(32, 400, 2), new=[min(12, n) for n in some(32, 400, 2)], page=32, missing=2),
    "missing_64": dict(B=16, Hq=64, H=32, T=9, lens=[200 + 9 * i for i in range(16)], new=None, page=64, missing=1),
    "missing_128": dict(B=16, Hq=64, H=32, T=10, lens=[500 - 13 * i for i in range(16)], new=[i % 11 for i in range(16)], page=128, missing=1),
    "all_missing": dict(B=64, Hq=8, H=8, T=17, lens=[64 + i for i in range(64)], new=None, page=16, missing=40),
    "docs": dict(B=64, Hq=8, H=8, T=18, lens=[150] * 64, new=None, page=16, masks="docs"),
    "window": dict(B=64, Hq=16, H=8, T=30, lens=[100 + 2 * i for i in range(64)], new=[30, 1, 0, 17] * 16, page=16, masks="window", missing=1),
    "holes": dict(B=64, Hq=8, H=8, T=25, lens=[120 + i for i in range(64)], new=None, page=32, masks="holes"),
    "both_ways": dict(B=128, Hq=4, H=4, T=20, lens=[20 + i for i in range(128)], new=None, page=64, masks="both_ways"),
    "eight_heads": dict(B=64, Hq=64, H=8, T=3, lens=[33 + 4 * i for i in range(64)], new=[3, 2, 1, 0] * 16, page=16),
    "three_tiles": dict(B=3, Hq=64, H=64, T=600, lens=[600, 40, 0], new=[600, 9, 0], page=16, missing=2),
    "many_pages": dict(B=2, Hq=256, H=256, T=20, lens=[2300, 1090], new=[3, 1], page=16, missing=9),
    "beyond_the_table": dict(B=64, Hq=8, H=8, T=20, lens=[90 + i for i in range(64)], new=None, page=16, width=6),
    "negative": dict(B=64, Hq=8, H=8, T=20, lens=[-2 ** 31, 10, -1, 40] * 16, new=None, page=16),
}


def run(rk, x, strided):  # noqa: F811
    geom, pages, q, table, lens, args = x.device(rk, strided=strided)
    assert x.B * x.H * -(-x.T * x.G // 256) >= 512 and x.T * x.G > 16 and not x.cap and x.slopes is None
    out, lse = x.blank()
    rk.rk_paged_attn(geom, q, pages, table, lens, x.width * x.page, out, lse=lse, workspace=rk.PromptWorkspace(geom, x.T, x.width * x.page), **args)
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.parametrize("name", list(CASES))
def test_wide(rk, name):  # noqa: F811
    say("paged, 64 rows to a wavefront", name)
    x = Inputs(**CASES[name])
    out, lse = run(rk, x, True)
    again = run(rk, x, False)
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
    if name == "three_tiles":
        x.H, x.Hq = 2, 2                                                         # (two heads of 64)
        x.q = x.q[:, :, :2]
        assert (out[1, 9:] == 9).all() and (out[2] == 9).all()
        out, lse = out[:, :, :2], lse[:, :, :2]
    x.check(out, lse, False, name)


@pytest.mark.parametrize("name", ["missing", "missing_64", "docs", "window", "holes", "eight_heads"])
def test_rows_that_a_token_does_not_see_have_no_part(rk, name):  # noqa: F811
    """Infinities and NaN planted in V: tokens that do not see them get what they get without, tokens that do get what comes of it."""
    say("planted, 64 rows to a wavefront", name)
    x = Inputs(**CASES[name])
    r = np.random.default_rng(1)
    clean, planted = x.V.clone(), []
    for b in range(x.B):
        n, s, there = o.places(x.table[b], x.page, x.n_pages, x.lens[b])
        for j in sorted(set(r.integers(0, x.lens[b], 3).tolist()) | {x.lens[b] - 1}):
            g, d, v = int(r.integers(x.H)), int(r.integers(128)), [math.inf, -math.inf, math.nan][int(r.integers(3))]
            if there[j]:
                x.V[n[j], g, s[j], d] = v
                planted.append((b, g, j, d, v))
    dirty, outs = x.V, []
    for x.V in (clean, dirty):
        out, lse = run(rk, x, False)
        outs.append((out.double().cpu().numpy(), lse.double().cpu().numpy()))
    (a, la), (c, lc) = outs
    x.V = clean
    assert (la == lc).all() and len(planted) > x.B
    seen_by = 0
    for b in range(x.B):
        for g in range(x.H):
            mine = [p for p in planted if p[:2] == (b, g)]
            hs = slice(g * x.G, (g + 1) * x.G)
            if not mine:
                assert (a[b, :, hs] == c[b, :, hs]).all(), (name, b, g)
                continue
            there = x.rows(b, g)[2]
            for i in range(x.new[b]):
                seen = set(x.seen(b, i, g, there)[1].tolist())
                want = a[b, i, hs].copy()
                for _, _, j, d, v in mine:
                    if j in seen:
                        with np.errstate(invalid="ignore"):                      # (infinities of both signs)
                            want[:, d] += v
                        seen_by += 1
                np.testing.assert_array_equal(c[b, i, hs], want, err_msg=str((name, b, i, g)))
    assert seen_by
