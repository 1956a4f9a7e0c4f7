"""rk_prompt_attn with caps of every size, far below the scores and far above them, against oracle/new_tokens.py."""
import math
import sys

import numpy as np
import pytest
import torch

from oracle import new_tokens as o

pytestmark = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))

SHAPES = {
    # B, Hq, Hkv, n_new, lens: each kernel and form that scores go through
    "columns": (1, 8, 2, 1, [700]),
    "columns_alone": (32, 8, 2, 1, [(37 * i) % 300 + 1 for i in range(32)]),
    "drafted": (2, 8, 4, 3, [260, 90]),
    "rows": (2, 8, 2, 70, [200, 70]),
    "rows_split": (1, 2, 1, 40, [3000]),
}


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def run(rk, shape, spread, cap, slopes, seed=11):
    B, Hq, H, T, lens = SHAPES[shape]
    g, rows = torch.Generator().manual_seed(seed), max(lens)
    q = (torch.randn(B, T, Hq, 128, generator=g) * spread).to(torch.bfloat16)
    q[0, 0, 0] = 0                                                               # a head whose products are all 0
    K, V = (torch.randn(B, H, rows, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    sl = torch.exp2(-torch.arange(1, Hq + 1).float()) if slopes else None
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    out, lse = torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, T, Hq, device="cuda")
    rk.rk_prompt_attn(geom, q.cuda(), K.cuda(), V.cuda(), torch.tensor(lens, dtype=torch.int32, device="cuda"), rows, out, lse=lse, cap=cap,
                      slopes=None if sl is None else sl.cuda(), workspace=rk.PromptWorkspace(geom, T, rows))
    return q, K, V, sl, out.double().cpu().numpy(), lse.double().cpu().numpy()


def check(shape, q, K, V, sl, cap, out, lse):
    """Scores: 128 products added in fp32 and five roundings around them, 140 * 2^-24 of their terms' sizes; of the cap's tanh 2^-19 of the score, or, where
    the cap is at most 128, 2^-22 of it at the most: no part that grows with a larger cap.  Weights: twice that, 2^-20, 2^-22 of s - max; in the product
    with V 2^-8 where they are bf16 (more than 16 rows of a group), 2^-16 otherwise.  The output is rounded once, 2^-8."""
    B, Hq, H, T, lens = SHAPES[shape]
    G = Hq // H
    qf, Kf, Vf = (x.double().numpy() for x in (q, K, V))
    for b in range(B):
        for i in sorted({0, T // 2, T - 1}):
            p = lens[b] - T + i
            for h in range(Hq):
                s1 = 0.0 if sl is None else float(sl[h])
                k, v = Kf[b, h // G, :p + 1], Vf[b, h // G, :p + 1]
                want, wl = o.prompt_attn(qf[b, i, h], Kf[b, h // G], Vf[b, h // G], p, 0, p + 1, SCALE, cap, s1)
                far = s1 * np.abs(p - np.arange(p + 1))
                c = cap * np.tanh(SCALE * (k @ qf[b, i, h]) / cap)
                ds = (140 * 2.0 ** -24 * (SCALE * (np.abs(k) @ np.abs(qf[b, i, h])) + far) + (2.0 ** -22 * cap if cap <= 128 else 2.0 ** -19 * np.abs(c))).max()
                s = c - far
                w = np.exp(s - s.max())
                w /= w.sum()
                rel = 2 * ds + 2.0 ** -20 + 2.0 ** -22 * np.abs(s - s.max()) + (2.0 ** -16 if T * G <= 16 else 2.0 ** -8)
                at = (shape, cap, b, i, h)
                assert abs(lse[b, i, h] - wl) <= ds + 2.0 ** -20 + 2.0 ** -22 * abs(wl), (at, lse[b, i, h], wl)
                err = np.abs(out[b, i, h] - want)
                assert (err <= 2.0 ** -8 * np.abs(want) + (rel * w) @ np.abs(v)).all(), (at, err.max())


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", [1e-42, 1e-30, 0.01, 30.0, 128.0, 129.0, 1e4, 1e6, 1e9, 3e38])
@pytest.mark.parametrize("shape", SHAPES)
def test_scores_of_ordinary_size(rk, shape, cap, slopes):
    print("caps", shape, cap, slopes, file=sys.stderr, flush=True)
    q, K, V, sl, out, lse = run(rk, shape, 3.0, cap, slopes)
    check(shape, q, K, V, sl, cap, out, lse)


@pytest.mark.parametrize("slopes", [False, True])
@pytest.mark.parametrize("cap", [100.0, 150.0, 300.0, 1000.0])
@pytest.mark.parametrize("shape", SHAPES)
def test_scores_of_the_caps_size(rk, shape, cap, slopes):
    """Scores of a few hundredths of the cap to about twice it, on both sides of where the series ends."""
    print("caps reached", shape, cap, slopes, file=sys.stderr, flush=True)
    q, K, V, sl, out, lse = run(rk, shape, cap / 2, cap, slopes)
    check(shape, q, K, V, sl, cap, out, lse)


@pytest.mark.parametrize("shape", SHAPES)
def test_a_cap_far_above_all_scores_is_none(rk, shape):
    print("caps none", shape, file=sys.stderr, flush=True)
    plain, far = run(rk, shape, 1.0, 0.0, False), run(rk, shape, 1.0, 1e30, False)
    # the same scores but for 2^-22 of themselves (6 at the most), weights 2^-18 apart, which may move the roundings of a weight and of the output, 2^-8 each,
    # either way (values of V below 6); log-sum-exps (up to 8) with 2^-20 and 2^-22 of themselves on either side
    assert (np.abs(plain[4] - far[4]) <= 4 * 2.0 ** -8 * 6).all() and np.abs(plain[5] - far[5]).max() <= 2.0 ** -17
    assert math.isfinite(far[5].max())
