"""rk_full_attn_q8 where a workgroup has all rows of a (sequence, KV head): against oracle/new_tokens.py."""
import math
import sys

import numpy as np
import pytest
import torch

from test_gpu_q8_attn import check, make

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))

CASES = [
    # name, B, Hq, H, block, format, lens, capacity
    ("g4", 8, 16, 4, 32, "e4m3", [500, 1, 0, 33, 511, 512, 320, 31], 512),
    ("g7_int8", 8, 28, 4, 16, "int8", [17, 500, 16, 15, 512, 0, 47, 333], 512),
    ("g8_block128", 16, 16, 2, 128, "e4m3", [(37 * i) % 513 for i in range(16)], 512),
    ("g1", 32, 1, 1, 64, "int8", [(61 * i) % 500 for i in range(32)], 512),
    ("longer_rounds", 32, 16, 8, 32, "e4m3", [(409 * i) % 2049 for i in range(32)], 2048),
    ("more_than_are_shared_out", 66, 12, 4, 32, "int8", [(1031 * i) % 2049 for i in range(66)], 2048),
    ("beyond_the_capacity", 33, 2, 1, 32, "e4m3", [600] * 33, 512),
]


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


@pytest.mark.parametrize("width", [0, 3], ids=["whole_lines", "odd_rows"])
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_attn(rk, case, width):
    name, B, Hq, H, block, fmt, lens, cap = case
    print("alone", name, width, file=sys.stderr, flush=True)
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    cache, rows = make(rk, 11, B, H, cap, block, fmt, lens, powers=width == 0, strided=width != 0)
    cache = cache(geom)
    q = torch.randn(B, Hq, 128, generator=torch.Generator().manual_seed(12)).to(torch.bfloat16)
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pred = torch.tensor([i % 9 != 4 for i in range(B)], dtype=torch.int32, device="cuda")
    ws = rk.Workspace(geom, cap, 1)
    new = lambda: (torch.full((B, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, Hq), 9.0, device="cuda"))  # noqa: E731
    (out, lse), (out2, lse2), w = new(), new(), torch.full((B, Hq, cap + width), -7.0, device="cuda")
    rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, cap, out, weights=w, lse=lse, pred=pred, pred_val=1, workspace=ws)
    rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, cap, out2, lse=lse2, pred=pred, pred_val=1, workspace=ws)
    torch.cuda.synchronize()
    assert torch.equal(out, out2) and torch.equal(lse, lse2)                     # with weights or without
    a, l, wn = out.double().cpu().numpy(), lse.double().cpu().numpy(), w.double().cpu().numpy()
    for b, m in enumerate(lens):
        if b % 9 == 4:
            assert (a[b] == 9).all() and (l[b] == 9).all() and (wn[b] == -7).all()
            continue
        m = min(m, cap)
        for h in range(Hq) if B <= 16 or b % 5 == 0 else (0, Hq - 1):
            check(q, rows, SCALE, b, Hq // H, h, m, a, l, wn, (name, b, h))
        assert (wn[b, :, m:] == -7).all()


@pytest.mark.parametrize("n_b,hq,h", [(65, 8, 4), (129, 4, 4)])
def test_longer_ones_of_more_than_are_shared_out(rk, n_b, hq, h):
    """Beyond what a workgroup takes alone with its weights, and beyond two workgroups to a compute unit."""
    lens = [(1213 * i) % 2900 for i in range(n_b)]
    geom = rk.Geom(n_b, hq, h, 128, SCALE)
    cache, rows = make(rk, 15, n_b, h, 2912, 32, "e4m3", lens)
    cache = cache(geom)
    q = torch.randn(n_b, hq, 128, generator=torch.Generator().manual_seed(16)).to(torch.bfloat16)
    sl, ws = torch.tensor(lens, dtype=torch.int32, device="cuda"), rk.Workspace(geom, 2912, 1)
    for weights in (None, torch.zeros(n_b, hq, 2912, device="cuda")):
        out, lse = torch.full((n_b, hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((n_b, hq), 9.0, device="cuda")
        rk.rk_full_attn_q8(geom, q.cuda(), cache, sl, 2912, out, weights=weights, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        a, l, wn = out.double().cpu().numpy(), lse.double().cpu().numpy(), None if weights is None else weights.double().cpu().numpy()
        for b in range(0, n_b, 8):
            for x in (0, hq - 1):
                check(q, rows, SCALE, b, hq // h, x, lens[b], a, l, wn, (weights is None, b, x))


def test_max_len_captured_and_a_nan_block(rk):
    B, Hq, H, cap, block = 32, 8, 2, 512, 32
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    lens = [(97 * i) % 513 for i in range(B)]
    cache, rows = make(rk, 13, B, H, cap, block, "e4m3", [512] * B)
    cache = cache(geom)
    q = torch.randn(B, Hq, 128, generator=torch.Generator().manual_seed(14)).to(torch.bfloat16)
    qd, sl, ws = q.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), rk.Workspace(geom, cap, 1)
    held, out = (torch.full((B, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    hw, w = torch.zeros(B, Hq, cap, device="cuda"), torch.zeros(B, Hq, cap, device="cuda")
    lse = torch.zeros(B, Hq, device="cuda")
    # no more than max_len rows (a step over full blocks of a cache that is filled further: what lies behind is not looked at)
    rk.rk_full_attn_q8(geom, qd, cache, torch.full_like(sl, 512), 96, out, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    a, l = out.double().cpu().numpy(), lse.double().cpu().numpy()
    for b in range(0, B, 7):
        for h in range(Hq):
            check(q, lambda n, b_, g, m: rows(n, b_, g, 512)[:96], SCALE, b, Hq // H, h, 96, a, l, None, ("max_len", b, h))
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        rk.rk_full_attn_q8(geom, qd, cache, sl, cap, held, weights=hw, workspace=ws)
    for step in range(3):
        sl.copy_(torch.tensor([(m + 32 * step) // 32 * 32 % 513 for m in lens], dtype=torch.int32))      # (some of them 31 rows: a tail of NaN)
        for t in (hw, w):
            t.zero_()
        graph.replay()
        rk.rk_full_attn_q8(geom, qd, cache, sl, cap, out, weights=w, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(held.view(torch.int16), out.view(torch.int16)) and torch.equal(hw.view(torch.int32), w.view(torch.int32)), step      # (bits: NaN too)
    cache.k_scale[3, 1, 4] = math.nan
    cache.v_scale[5, 0, 0] = math.nan
    sl.fill_(512)
    rk.rk_full_attn_q8(geom, qd, cache, sl, cap, out, weights=w, lse=lse, workspace=ws)
    torch.cuda.synchronize()
    G = Hq // H
    assert out[3, G:].isnan().all() and lse[3, G:].isnan().all() and w[3, G:].isnan().all() and not out[3, :G].isnan().any()
    assert out[5, :G].isnan().all() and not lse[5].isnan().any() and not out[4].isnan().any()
