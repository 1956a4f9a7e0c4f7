"""Arguments of the calls over pages that Python refuses: host numbers beyond 32 bits, which the C calls would get without their upper bits, and what is no tensor."""
import pytest
import torch

BIG = 2 ** 32 + 16


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


@pytest.mark.parametrize("sizes", [(BIG, 64, 64), (1, BIG, 64), (1, 64, BIG), (1, 64, -BIG)])
def test_workspaces(rk, sizes):
    geom = rk.Geom(1, 4, 2, 128, 0.1)
    with pytest.raises(ValueError):
        rk.PrefixWorkspace(geom, *sizes, device="cpu")
    with pytest.raises(ValueError):
        rk.SparseWorkspace(geom, *sizes, device="cpu")


@pytest.mark.gpu
def test_calls(rk):
    geom = rk.Geom(1, 4, 2, 128, 0.1)
    pool, i32 = rk.Pages.empty(geom, 8, 16), lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, lens, q = i32([list(range(8))]), i32([100]), torch.zeros(1, 1, 4, 128, dtype=torch.bfloat16, device="cuda")
    out, scores, idx = torch.full_like(q, 9.0), torch.full((1, 1, 2, 8), 9.0, device="cuda"), torch.full((1, 1, 2, 4), 9, dtype=torch.int32, device="cuda")
    pws, xws, sws = rk.PromptWorkspace(geom, 1, 128), rk.PrefixWorkspace(geom, 1, 32, 128), rk.SparseWorkspace(geom, 1, 4, 16)

    def prefix(pt=table[0, :2].contiguous(), pl=i32([32]), most=32, own=96):
        rk.rk_prefix_attn(geom, q, pool, pt, pl, most, table, lens, own, out, workspace=xws)

    def select(s=scores, page=16, k=4, to=idx, **kw):
        rk.rk_page_select(geom, s, page, lens, k, to, **kw)
    bad = [lambda: prefix(own=BIG), lambda: prefix(most=BIG), lambda: prefix(most=-BIG), lambda: prefix(pt=None), lambda: prefix(pl=None),
           lambda: rk.rk_paged_attn(geom, q, pool, table, lens, -BIG, out, workspace=pws), lambda: rk.rk_page_scores(geom, q, pool, table, lens, None),
           lambda: rk.rk_page_scores(geom, q, pool, table, lens, scores, agg=2 ** 32), lambda: select(page=BIG), lambda: select(k=2 ** 32 + 4), lambda: select(s=None), lambda: select(to=None),
           lambda: select(keep_first=2 ** 32), lambda: select(keep_last=2 ** 32 + 1), lambda: rk.rk_sparse_attn(geom, q, pool, table, None, lens, out, workspace=sws),
           lambda: rk.rk_paged_attn(geom, q, pool, table, lens, 128, out, workspace=pws, pred=i32([0]), pred_val=2 ** 32)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail(str(i))
    torch.cuda.synchronize()
    assert (out == 9).all() and (scores == 9).all() and (idx == 9).all()
    prefix()
    select(keep_first=2 ** 31 - 1, keep_last=2 ** 31 - 1)
    torch.cuda.synchronize()
    assert (out == 0).all() and idx[0, 0, 0].tolist() == [0, 1, 2, 3]
