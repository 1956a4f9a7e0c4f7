"""Calls over pages with room for 2^24 rows of queries and more, of which few are there: the same results as from calls with room for these alone, and
nothing else written."""
import pytest
import torch

from test_gpu_paged_attn import SCALE, i32, rk, say  # noqa: F401

pytestmark = pytest.mark.gpu

B, Hq, H, T, FEW, PAGE, N = 64, 32, 8, 8192, 40, 16, 128
NEW = [(7 * b) % (FEW + 1) for b in range(B)]


def enough():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GiB")


@pytest.fixture(scope="module")
def pool(rk):  # noqa: F811
    g = torch.Generator(device="cuda").manual_seed(2)
    K, V = (torch.randn(B * N // PAGE, H, PAGE, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    table = torch.randperm(B * N // PAGE, generator=g, device="cuda").view(B, -1).int()
    q = torch.randn(B, FEW, Hq, 128, generator=g, device="cuda").to(torch.bfloat16)
    return rk.Geom(B, Hq, H, 128, SCALE), rk.Pages(K, V), table, q, i32([N - b % 50 for b in range(B)]), i32(NEW)


@pytest.mark.parametrize("kind", ["paged", "sparse", "prefix"])
def test_attentions(rk, pool, kind):  # noqa: F811
    say("room for many rows", kind)
    enough()
    geom, pages, table, q, lens, new = pool
    idx = torch.randint(0, N // PAGE, (B, FEW, H, 3), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    if kind == "prefix":                                                         # everybody's first rows are the first sequence's
        table = table.clone()
        table[:, :2] = table[0, :2]
    res = []
    for n in (FEW, T):
        qn = torch.zeros(B, n, Hq, 128, dtype=torch.bfloat16, device="cuda")
        qn[:, :FEW] = q
        out, lse = torch.full_like(qn, 9.0), torch.full((B, n, Hq), 9.0, device="cuda")
        if kind == "paged":
            rk.rk_paged_attn(geom, qn, pages, table, lens, N, out, new_lens=new, lse=lse, workspace=rk.PromptWorkspace(geom, n, N))
        elif kind == "sparse":
            ix = torch.zeros(B, n, H, 3, dtype=torch.int32, device="cuda")
            ix[:, :FEW] = idx
            rk.rk_sparse_attn(geom, qn, pages, table, ix, lens, out, new_lens=new, lse=lse, workspace=rk.SparseWorkspace(geom, n, 3, PAGE))
        else:
            rk.rk_prefix_attn(geom, qn, pages, table[0, :2].contiguous(), i32([30]), 30, table, lens, N, out, new_lens=new, lse=lse, workspace=rk.PrefixWorkspace(geom, n, 30, N))
        torch.cuda.synchronize()
        assert n == FEW or bool((out[:, FEW:] == 9).all() and (lse[:, FEW:] == 9).all())
        res.append((out[:, :FEW].clone(), lse[:, :FEW].clone()))
        del qn, out, lse
    # weights as bf16 on both sides, at most 2^-8 of the values' size each, and half a step of the output's; sums and their order in fp32
    (a, la), (c, lc) = res
    there = torch.arange(FEW, device="cuda")[None] < new[:, None]
    assert (c[~there] == 9).all() and (lc[~there] == 9).all()
    assert (a.double() - c.double()).abs().max() <= 4 * 2.0 ** -8 * float(pages.v.abs().max())
    none = la == -float("inf")                                                   # (tokens whose chosen pages lie behind them)
    assert torch.equal(none, lc == -float("inf")) and (la - lc).masked_fill(none, 0.0).abs().max() <= 1e-4
    if kind != "prefix":
        b = next(i for i in range(B) if NEW[i])
        p = int(lens[b]) - NEW[b]
        rows = torch.arange(N, device="cuda")
        K, V = (y[table[b].long(), 0].reshape(N, 128).double() for y in (pages.k, pages.v))
        s = SCALE * K @ q[b, 0, 0].double()
        seen = rows <= p
        if kind == "sparse":
            seen = seen & (rows[:, None] // PAGE == idx[b, 0, 0]).any(dim=1)
            s = s + torch.log((rows[:, None] // PAGE == idx[b, 0, 0]).sum(dim=1).clamp(min=1).double())      # (a page that is there twice counts twice)
        s = s.masked_fill(~seen, -float("inf"))
        want = torch.softmax(s, 0) @ V
        assert (c[b, 0, 0].double() - want).abs().max() <= 2 * 2.0 ** -8 * float(V.abs().max())


def test_selection(rk):  # noqa: F811
    say("room for many rows of scores")
    enough()
    b, t, n, k, page, few = 16, 32768, 41, 5, 128, 100
    geom = rk.Geom(b, Hq, H, 128, SCALE)
    scores = torch.randn(b, t, H, n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    lens, new = [n * page - 90 * x for x in range(b)], [few - x for x in range(b)]
    idx = torch.full((b, t, H, k), 77, dtype=torch.int32, device="cuda")
    rk.rk_page_select(geom, scores, page, i32(lens), k, idx, new_lens=i32(new), keep_first=1, keep_last=1)
    for x in range(b):
        own = (torch.arange(new[x], device="cuda") + lens[x] - new[x]) // page
        s, j = scores[x, :new[x]].clone(), torch.arange(n, device="cuda")
        s[..., 0] = float("inf")
        s.masked_fill_((j == own[:, None])[:, None], float("inf"))
        s.masked_fill_((j > own[:, None])[:, None], -float("inf"))
        assert torch.equal(idx[x, :new[x]].long(), s.topk(k, dim=-1).indices.sort(dim=-1).values), x
        assert (idx[x, new[x]:] == 77).all()


@pytest.mark.parametrize("T", [2, 5, 30])
def test_a_wider_table_changes_no_bit(rk, T):  # noqa: F811
    """The form that keeps chosen rows in the caches and the one that passes them by, which a table's width decides between."""
    say("chosen pages of a wider table", T)
    geom, g = rk.Geom(3, 16, 4, 128, SCALE), torch.Generator().manual_seed(5)
    K, V = (torch.randn(3 * 20, 4, PAGE, 128, generator=g).to(torch.bfloat16).cuda() for _ in range(2))
    table, q = torch.randperm(60, generator=g).view(3, 20).int(), torch.randn(3, T, 16, 128, generator=g).to(torch.bfloat16).cuda()
    idx = torch.randint(0, 20, (3, T, 4, 6), generator=g, dtype=torch.int32).cuda()
    outs = []
    for width in (20, 4000):
        wide = torch.full((3, width), -1, dtype=torch.int32)
        wide[:, :20] = table
        out, lse = torch.zeros_like(q), torch.zeros(3, T, 16, device="cuda")
        rk.rk_sparse_attn(geom, q, rk.Pages(K, V), wide.cuda(), idx, i32([320, 300, 111]), out, lse=lse, workspace=rk.SparseWorkspace(geom, T, 6, PAGE))
        assert (2 * T * 6 >= width) == (width == 20)
        outs.append((out, lse))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_more_threads_than_32_bits_count(rk):  # noqa: F811
    """A token of as many sequences and KV heads as make 2^32 threads and more, along three axes: equal keys, so each output is the mean of the values seen."""
    say("2^32 threads")
    enough()
    b, h = 65535, 300
    assert b * h * 256 >= 1 << 32
    V = torch.arange(16, device="cuda").to(torch.bfloat16)[None, None, :, None].expand(1, h, 16, 128).contiguous()
    pool = rk.Pages(torch.zeros_like(V), V)
    q = torch.ones(b, 1, h, 128, dtype=torch.bfloat16, device="cuda")
    lens = torch.arange(b, device="cuda", dtype=torch.int32) % 16 + 1
    out = torch.full_like(q, 99.0)
    rk.rk_paged_attn(rk.Geom(b, h, h, 128, SCALE), q, pool, torch.zeros(b, 1, dtype=torch.int32, device="cuda"), lens, 16, out)
    torch.cuda.synchronize()
    want = ((lens - 1).float() / 2).to(torch.bfloat16)
    assert bool((out == want[:, None, None, None]).all())
