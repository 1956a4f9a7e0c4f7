"""Sequences that are longer than their table, whose rows behind it do not exist, and score rows that are wider than it: rk_page_scores leaves -infinity for
the pages that a token would see there, so that rk_page_select ranks nothing that an earlier call or nobody wrote."""
import math

import numpy as np
import pytest
import torch

from oracle import paged as o
from test_gpu_paged_attn import SCALE, i32, rk, say  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = {
    # B, Hq, Hkv, T, table width, wider by, page, rows behind the table (by sequence, in turn), new, agg
    "step": (1, 32, 8, 1, 5, 3, 16, [1], None, "max"),
    "a_row_behind": (2, 8, 2, 1, 64, 1, 16, [1, 0], None, "mean"),
    "steps": (3, 28, 4, 1, 65, 70, 64, [4000, -100, 64], None, "max"),
    "wider_than_seen": (2, 4, 4, 2, 20, 500, 32, [100, 2000], None, "first"),
    "longer_than_wide": (2, 8, 1, 3, 130, 9, 16, [5000, 2 ** 31 - 1 - 130 * 16], None, "max"),
    "across_the_end": (2, 16, 2, 40, 7, 20, 16, [25, 3], None, "max"),
    "ragged": (4, 10, 2, 30, 63, 90, 16, [400, 20, -300, 1500], [30, 7, 30, 0], "mean"),
    "no_wider": (2, 8, 2, 3, 30, 0, 16, [100, 20], None, "max"),
    "many_sequences": (33, 8, 8, 2, 40, 33, 16, [0, 9, 100, -50, 3000], None, "max"),
    "many_pages": (32, 8, 8, 3, 300, 100, 16, [700, -9, 1, 16, 5000], [3, 0, 2, 3, 1] * 6 + [3, 3], "mean"),
    "ends_with_a_wavefront": (32, 16, 8, 1, 256, 50, 32, [300, 31, 32], None, "first"),
    "many_tokens": (3, 7, 1, 300, 100, 64, 16, [150, 300, 2000], [300, 250, 3], "max"),
}


def wanted(lens, new, width, W, page, B, T):
    """What every entry is: 0 as it was, 1 a score, 2 -infinity."""
    kind = np.zeros((B, T, W), np.int64)
    for b in range(B):
        for i in range(new[b]):
            last = (lens[b] - new[b] + i) // page
            kind[b, i, :max(0, min(last + 1, W))] = 2
            kind[b, i, :max(0, min(last + 1, width, W))] = 1
    return kind


@pytest.mark.parametrize("name", list(CASES))
def test_scores_and_selection(rk, name):  # noqa: F811
    say("scores behind the table", name)
    B, Hq, H, T, width, wider, page, behind, new, agg = CASES[name]
    geom, W = rk.Geom(B, Hq, H, 128, SCALE), width + wider
    lens = [width * page + behind[b % len(behind)] for b in range(B)]
    nl = [T] * B if new is None else new
    g = torch.Generator().manual_seed(6)
    n_pages = B * width + 1
    table = torch.randperm(n_pages, generator=g)[:B * width].view(B, width).int().cuda()
    a, c = (torch.randn(n_pages, H, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    K = torch.zeros(n_pages, H, page, 128, dtype=torch.bfloat16, device="cuda")
    pool = rk.Pages(K, K, torch.minimum(a, c).cuda(), torch.maximum(a, c).cuda())
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16).cuda()
    agg = {"max": rk.RK_AGG_MAX, "mean": rk.RK_AGG_MEAN, "first": rk.RK_AGG_FIRST}[agg]
    left = 1e9                                                                   # what was there: better than any score
    out, just = torch.full((B, T, H, W), left, device="cuda"), torch.full((B, T, H, width), left, device="cuda")
    rk.rk_page_scores(geom, q, pool, table, i32(lens), out, new_lens=i32(new), agg=agg)
    rk.rk_page_scores(geom, q, pool, table, i32(lens), just, new_lens=i32(new), agg=agg)
    got, kind = out.cpu().numpy(), wanted(lens, nl, width, W, page, B, T)
    assert (kind == 2).any() == (wider > 0)
    for h in range(H):
        assert (got[:, :, h][kind == 0] == left).all() and (got[:, :, h][kind == 2] == -math.inf).all()
        assert np.isfinite(got[:, :, h][kind == 1]).all() and (got[:, :, h][kind == 1] < left).all()
    assert torch.equal(out[..., :width], just)
    # the pages with the largest: those that there are, as long as there are k of them
    k = min(4, width)
    idx = torch.full((B, T, H, k), 77, dtype=torch.int32, device="cuda")
    rk.rk_page_select(geom, out, page, i32(lens), k, idx, new_lens=i32(new), keep_first=1, keep_last=0)
    ix = idx.cpu().numpy()
    for b in range(B):
        assert (ix[b, nl[b]:] == 77).all()
        for i in range(nl[b]):
            last = (lens[b] - nl[b] + i) // page
            assert (ix[b, i] < width).all()
            for h in range(H):
                np.testing.assert_array_equal(ix[b, i, h], o.select(got[b, i, h], last, k, 1, 0), err_msg=str((name, b, i, h)))
