"""rk_prompt_attn where a sequence's length is no number of rows: negative, down to the lowest, as an idle slot of a batch may have it."""
import math
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu
LOW = -2 ** 31


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


@pytest.mark.parametrize("form", ["", "slopes", "cap", "ranges"])
@pytest.mark.parametrize("T", [1, 2, 3, 70])
@pytest.mark.parametrize("length", [LOW, LOW + 1, -70, -1, 0])
def test_nothing_is_seen(rk, length, T, form):
    """Its tokens see no row: 0 and -inf; the sequence beside it is as it is alone.  (A token's position, the length less up to 70, lies below 32 bits.)"""
    print("length", length, T, form, file=sys.stderr, flush=True)
    Hq, H, rows = 8, 2, 300
    g = torch.Generator().manual_seed(5)
    q = torch.randn(2, T, Hq, 128, generator=g).to(torch.bfloat16).cuda()
    K, V = (torch.randn(2, H, rows, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    more = {}
    if form == "slopes":
        more["slopes"] = torch.full((Hq,), 0.1, device="cuda")
    if form == "cap":
        more["cap"] = 20.0
    if form == "ranges":
        more["first"], more["end"] = (torch.full((2, T), x, dtype=torch.int32, device="cuda") for x in (LOW, 2 ** 31 - 1))
    outs = []
    for lens in ([length, 200], [200, length]):
        geom = rk.Geom(2, Hq, H, 128, 0.1)
        out, lse = torch.full_like(q, 9.0), torch.full((2, T, Hq), 9.0, device="cuda")
        rk.rk_prompt_attn(geom, q, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows, out, lse=lse, workspace=rk.PromptWorkspace(geom, T, rows), **more)
        torch.cuda.synchronize()
        outs.append((out, lse))
    (a, la), (b, lb) = outs
    assert (a[0] == 0).all() and (la[0] == -math.inf).all() and (b[1] == 0).all() and (lb[1] == -math.inf).all()
    assert a[1].isfinite().all() and la[1].isfinite().all() and b[0].isfinite().all() and lb[0].isfinite().all()
    for x, (got, gl) in ((1, outs[0]), (0, outs[1])):                            # the other one, in a batch whose neighbour has no rows either way
        geom, lens = rk.Geom(2, Hq, H, 128, 0.1), [0, 0]
        lens[x] = 200
        out, lse = torch.zeros_like(q), torch.zeros(2, T, Hq, device="cuda")
        rk.rk_prompt_attn(geom, q, K, V, torch.tensor(lens, dtype=torch.int32, device="cuda"), rows, out, lse=lse, workspace=rk.PromptWorkspace(geom, T, rows), **more)
        assert torch.equal(out[x], got[x]) and torch.equal(lse[x], gl[x])
