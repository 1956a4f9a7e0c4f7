"""The calls around the decode step as a server makes them: prompts in, a cache of 8 bits, full steps, refreshes and partial steps out of it; captured,
over caches past 32 bits, through either marshalling."""
import math
import sys

import numpy as np
import pytest
import torch

import gen
from oracle import new_tokens as o
from oracle import steps
from test_gpu_prompt_attn import close
from test_gpu_q8_attn import check

gpu = pytest.mark.gpu
SCALE = float(np.float32(1 / np.sqrt(128)))


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


def say(*a):
    print(*a, file=sys.stderr, flush=True)


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@gpu
@pytest.mark.parametrize("fmt,block", [("e4m3", 32), ("int8", 16)])
def test_a_served_run(rk, fmt, block):
    """Two ragged prompts in chunks, then decode steps: every fourth one full, with a refresh of the small cache from its scores."""
    say("served run", fmt, block)
    B, Hq, H, cap, n_sel, pool, stride = 2, 8, 2, 512, 64, 7, 4
    G, geom = Hq // H, rk.Geom(B, Hq, H, 128, SCALE)
    bf = dict(dtype=torch.bfloat16, device="cuda")
    gen_ = torch.Generator().manual_seed(17)
    chunks = [[130, 90], [60, 0], [1, 85]]                                       # new tokens of each sequence, call by call
    rope = rk.Rope(rk.rope_table(cap, 128, base=500000.0, factor=8.0, low_turns=1.0, high_turns=4.0, original_len=8192))
    K, V = (torch.zeros(B, H, cap, 128, **bf) for _ in range(2))                 # the prompts' rows, bf16
    cache = rk.Kv8.empty(geom, cap, block, torch.float8_e4m3fn if fmt == "e4m3" else torch.int8)
    lens = np.zeros(B, np.int32)
    pws = rk.PromptWorkspace(geom, 130, cap)
    for new in chunks:
        T = max(new)
        w = torch.randn(B, T, Hq + 2 * H, 128, generator=gen_).to(torch.bfloat16).cuda()
        q, k, v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
        lens = lens + np.array(new, np.int32)
        sl, nl = i32(lens.tolist()), i32(new)
        qo, out, lse = torch.zeros(B, T, Hq, 128, **bf), torch.full((B, T, Hq, 128), 9.0, **bf), torch.full((B, T, Hq), 9.0, device="cuda")
        rk.rk_rope_append(geom, q, k, v, rope, K, V, sl, qo, new_lens=nl)
        rk.rk_rope_append_q8(geom, None, k, v, rope, cache, sl, None, new_lens=nl)
        rk.rk_prompt_attn(geom, qo, K, V, sl, cap, out, new_lens=nl, lse=lse, workspace=pws)
        torch.cuda.synchronize()
        case = ("prompt", B, Hq, H, T, lens.tolist(), new, "causal", 0.0, False)
        close(case, geom, qo.cpu(), K.cpu(), V.cpu(), new, None, None, None, out, lse)
    Kn, Vn = gen.bf16_bits(K.cpu()), gen.bf16_bits(V.cpu())
    held = [[[o.Cache8(block, fmt) for _ in range(2)] for _ in range(H)] for _ in range(B)]
    for b in range(B):
        for h in range(H):
            for x, rows in zip(held[b][h], (Kn, Vn)):
                for r in range(lens[b]):
                    x.append(rows[b, h, r])

    ws = rk.Workspace(geom, cap, n_sel)
    rK, rV = (torch.zeros(B, H, n_sel + stride, 128, **bf) for _ in range(2))    # the small cache, and behind it the tokens since the refresh
    sK, sV = rK[:, :, :n_sel], rV[:, :, :n_sel]
    idx, zero = torch.zeros(B, H, n_sel, dtype=torch.int32, device="cuda"), i32([0] * B)
    weights, lse = torch.zeros(B, Hq, cap, device="cuda"), torch.zeros(B, Hq, device="cuda")
    for t in range(3 * stride):
        w = torch.randn(B, 1, Hq + 2 * H, 128, generator=gen_).to(torch.bfloat16).cuda()
        q, k, v = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
        lens = lens + 1
        sl, since = i32(lens.tolist()), t % stride
        qo, out = torch.zeros(B, 1, Hq, 128, **bf), torch.zeros(B, Hq, 128, **bf)
        rk.rk_rope_append_q8(geom, q, k, v, rope, cache, sl, qo)
        row_k, row_v = (torch.zeros(B, H, 1, 128, **bf) for _ in range(2))
        rk.rk_rope_append(geom, None, k, v, rope, row_k, row_v, zero + 1, None, positions=(sl - 1)[:, None].contiguous())
        for b in range(B):
            for h in range(H):
                for x, row in zip(held[b][h], (row_k, row_v)):
                    x.append(gen.bf16_bits(row.cpu())[b, h, 0])
        rows = lambda n, b, h, m: held[b][h]["kv".index(n)].rows()  # noqa: E731
        q1 = qo[:, 0]
        if since == 0:
            rk.rk_full_attn_q8(geom, q1, cache, sl, cap, out, weights=weights, lse=lse, workspace=ws)
            rk.rk_topk_select(geom, weights, sl, cap, n_sel, pool, idx, workspace=ws)
            rk.rk_gather_small_kv_q8(geom, cache, idx, n_sel, sK, sV, sl)
            torch.cuda.synchronize()
            a, l, wn = out.double().cpu().numpy(), lse.double().cpu().numpy(), weights.double().cpu().numpy()
            for b in range(B):
                for h in range(Hq):
                    check(q1.cpu(), rows, SCALE, b, G, h, int(lens[b]), a, l, wn, (t, b, h))
            sel, _ = steps.topk_select(weights.cpu().numpy(), lens, H, n_sel, pool)
            assert np.array_equal(idx.cpu().numpy(), sel)                         # from the same weights: the same rows
            for b in range(B):
                for h in range(H):
                    for n, got in (("k", sK), ("v", sV)):
                        assert np.array_equal(gen.bf16_bits(got.cpu())[b, h], o.f64_to_bf16_bits(rows(n, b, h, 0)[sel[b, h]])), (t, b, h)
            continue
        # a partial step: the small cache and what came since
        rk.rk_rope_append(geom, None, k, v, rope, rK, rV, zero + n_sel + since, None, positions=(sl - 1)[:, None].contiguous())
        rk.rk_partial_attn(geom, q1, sK, sV, n_sel, rK, rV, zero + n_sel, zero + n_sel + since, stride, out, workspace=ws)
        torch.cuda.synchronize()
        bits = [gen.bf16_bits(x.cpu()) for x in (q1, sK, sV, rK, rV)]
        want = o.bf16_bits_to_f64(steps.partial_attn(*bits[:3], n_sel, *bits[3:], np.full(B, n_sel, np.int32), np.full(B, n_sel + since, np.int32), SCALE))
        # both sides are rounded to bf16, and the weights are kept to 2^-16 or better: a step of 2^-7 and 2^-15 of the largest value
        assert (np.abs(out.double().cpu().numpy() - want) <= 2.0 ** -7 * np.abs(want) + 2.0 ** -15 * 448).all(), t


@gpu
@pytest.mark.parametrize("T", [1, 3, 40])
@pytest.mark.parametrize("scale", [-SCALE, 0.0])
@pytest.mark.parametrize("cap,slopes", [(0.0, False), (4.0, False), (0.0, True), (4.0, True)])
def test_scales_below_and_at_zero(rk, T, scale, cap, slopes):
    """A negative scale turns the order of the scores around; with 0 all rows that are seen weigh alike, but for the bias."""
    B, Hq, H, lens, new = 2, 8, 2, [700, 90], [T, max(T - 1, 1)]
    geom = rk.Geom(B, Hq, H, 128, scale)
    g = torch.Generator().manual_seed(21)
    q = (torch.randn(B, T, Hq, 128, generator=g) * 2).to(torch.bfloat16)
    K, V = (torch.randn(B, H, 704, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    first = np.maximum(np.array(lens)[:, None] - np.array(new)[:, None] + np.arange(T) - 50, 0).astype(np.int32)
    end = (np.array(lens)[:, None] - np.array(new)[:, None] + np.arange(T) + 1).astype(np.int32)
    if T > 1:
        end[0, 1] = first[0, 1]                                                  # sees nothing
    sl = torch.exp2(-torch.arange(1, Hq + 1).float()) if slopes else None
    out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
    rk.rk_prompt_attn(geom, q.cuda(), K.cuda(), V.cuda(), i32(lens), 704, out, new_lens=i32(new), first=i32(first.tolist()), end=i32(end.tolist()), cap=cap,
                      slopes=None if sl is None else sl.cuda(), lse=lse, workspace=rk.PromptWorkspace(geom, T, 704))
    torch.cuda.synchronize()
    # (the tolerance takes the size of the terms, whatever the scale's sign)
    close(("scale", B, Hq, H, T, lens, new, "", cap, slopes), _AbsScale(geom), _signed(q, scale), K, V, new, first, end, sl, out, lse)


class _AbsScale:
    def __init__(self, geom):
        self.scale = abs(geom.scale)


def _signed(q, scale):
    return -q if scale < 0 else q


@gpu
@pytest.mark.parametrize("B", [64, 65])
def test_many_ragged_sequences_of_few_tokens(rk, B):
    """Shared out by length up to 64 sequences, evenly beyond; empty ones, and those that the predicate leaves alone."""
    Hq, H, T, cap = 4, 1, 2, 640
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(B)
    lens = [(i * 97) % 640 if i % 7 else 0 for i in range(B)]
    new = [min(m, T) if i % 5 else min(m, 1) for i, m in enumerate(lens)]
    q = torch.randn(B, T, Hq, 128, generator=g).to(torch.bfloat16)
    K, V = (torch.randn(B, H, cap, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    for b, m in enumerate(lens):
        K[b, :, m:], V[b, :, m:] = math.nan, math.nan
    pred = [1 if i % 11 else 0 for i in range(B)]
    out, lse = torch.full((B, T, Hq, 128), 9.0, dtype=torch.bfloat16, device="cuda"), torch.full((B, T, Hq), 9.0, device="cuda")
    rk.rk_prompt_attn(geom, q.cuda(), K.cuda(), V.cuda(), i32(lens), cap, out, new_lens=i32(new), lse=lse, pred=i32(pred), pred_val=1,
                      workspace=rk.PromptWorkspace(geom, T, cap))
    torch.cuda.synchronize()
    nl = [n if p else 0 for n, p in zip(new, pred)]                              # (the predicate's: as if they had no new tokens)
    at = [m - n + x for m, n, x in zip(lens, new, nl)]
    close(("ragged", B, Hq, H, T, at, nl, "causal", 0.0, False), geom, q, K, V, nl, None, None, None, out, lse)


@gpu
def test_two_captured_calls_share_a_workspace(rk):
    """A prompt in split row tiles and a decode step, two graphs over one workspace, replayed in turn between eager calls; lengths, ranges and the cache
    change between replays."""
    B, Hq, H, cap, T = 2, 8, 2, 4096, 30
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator(device="cuda").manual_seed(4)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    q, q1, K, V = rnd(B, T, Hq, 128), rnd(B, 1, Hq, 128), rnd(B, H, cap, 128), rnd(B, H, cap, 128)
    q8, cache = q1[:, 0].contiguous(), rk.Kv8.empty(geom, cap, 64)
    new = rnd(B, 100, Hq + 2 * H, 128)
    ws, own, dws = rk.PromptWorkspace(geom, T, cap), rk.PromptWorkspace(geom, T, cap), rk.Workspace(geom, cap, 1)
    sl, nl, first = i32([4000, 2500]), i32([T, 7]), torch.zeros(B, T, dtype=torch.int32, device="cuda")
    l8, n8 = i32([0, 0]), i32([0, 0])
    held, eager = ([torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, 1, Hq, 128, dtype=torch.bfloat16, device="cuda"),
                    torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hq, cap, device="cuda")] for _ in range(2))

    def prompt(o_, w):
        rk.rk_prompt_attn(geom, q, K, V, sl, cap, o_[0], new_lens=nl, first=first, cap=20.0, workspace=w)

    def step(o_, w):
        rk.rk_prompt_attn(geom, q1, K, V, sl, cap, o_[1], workspace=w)
        rk.rk_full_attn_q8(geom, q8, cache, l8, cap, o_[2], weights=o_[3], workspace=dws)

    def append():
        rk.rk_rope_append_q8(geom, None, new[:, :, Hq:Hq + H], new[:, :, Hq + H:], None, cache, l8, None, new_lens=n8)
    side = torch.cuda.Stream()
    graphs = []
    torch.cuda.synchronize()
    for body in (append, lambda: prompt(held, ws), lambda: step(held, ws)):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            body()
        graphs.append(graph)
    total = np.zeros(2, np.int64)
    for turn, (lens, toks, lo, add) in enumerate((([4000, 2500], [T, 7], 0, [100, 33]), ([4096, 1], [T, 1], 3900, [27, 100]), ([0, 64], [0, 30], 10, [1, 0]),
                                                  ([31, 4095], [29, 30], 0, [100, 64]))):
        sl.copy_(i32(lens)), nl.copy_(i32(toks)), first.fill_(lo)
        total += add
        l8.copy_(i32(total.tolist())), n8.copy_(i32(add))
        for t in (*held, *eager):
            t.zero_()
        for graph in graphs:
            graph.replay()
        prompt(eager, own)
        step(eager, own)
        torch.cuda.synchronize()
        for x, y in zip(held, eager):
            assert torch.equal(x, y), turn
        # (what the replayed append put there is what an eager one into another cache puts)
        if turn == 3:
            twin, at = rk.Kv8.empty(geom, cap, 64), np.zeros(2, np.int64)
            for a in ([100, 33], [27, 100], [1, 0], [100, 64]):
                at += a
                rk.rk_rope_append_q8(geom, None, new[:, :, Hq:Hq + H], new[:, :, Hq + H:], None, twin, i32(at.tolist()), None, new_lens=i32(a))
            torch.cuda.synchronize()
            for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail"):
                a, b = getattr(cache, n), getattr(twin, n)
                assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), n


@gpu
def test_caches_past_32_bits(rk):
    """Three KV heads of 2^23 rows: the last one's lie more than 2^32 bytes behind the first one's.  Append at the end, few tokens, a tile of tokens."""
    n, cap, H, G, T = (1 << 23) + 57, (1 << 23) + 64, 3, 2, 20
    geom = rk.Geom(1, H * G, H, 128, SCALE)
    K, V = (torch.zeros(1, H, cap, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    g = torch.Generator().manual_seed(9)
    k, v = (torch.randn(1, T, H, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    sl = i32([n])
    rk.rk_rope_append(geom, None, k.cuda(), v.cuda(), None, K, V, sl, None)
    torch.cuda.synchronize()
    assert torch.equal(K[0, :, n - T:n].cpu(), k[0].transpose(0, 1)) and torch.equal(V[0, :, n - T:n].cpu(), v[0].transpose(0, 1))
    assert not K[0, :, n:].any() and not V[0, :, n - T - 4096:n - T].any()
    # a token's query is its own key times 40: e^(40 |k|^2 scale) is far beyond the 2^23 rows of score 0
    q = (40 * k).repeat_interleave(G, dim=2).contiguous()
    for lo in (0, n - 300):
        for t in (1, T):                                                         # columns, row tiles
            out, lse = torch.zeros(1, t, H * G, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, t, H * G, device="cuda")
            first = torch.full((1, t), lo, dtype=torch.int32, device="cuda")
            rk.rk_prompt_attn(geom, q[:, T - t:].contiguous().cuda(), K, V, sl, cap, out, first=first, lse=lse, workspace=rk.PromptWorkspace(geom, t, cap))
            torch.cuda.synchronize()
            for i in range(t):
                p = T - t + i
                for h in range(H * G):
                    kd, qd = k[0, :p + 1, h // G].double(), q[0, p, h].double()
                    s = SCALE * (kd @ qd)
                    m = float(s.max())
                    want = m + math.log(float(torch.exp(s - m).sum()) + (n - T - lo) * math.exp(-m))
                    # 128 products added in fp32, and fp32's steps at scores of several hundred
                    assert abs(float(lse[0, i, h]) - want) <= 140 * 2.0 ** -24 * float(SCALE * (kd[p].abs() @ qd.abs())) + 2.0 ** -21 * abs(want), (lo, t, i, h)
                    assert torch.equal(out[0, i, h].cpu(), v[0, p, h // G]), (lo, t, i, h)      # (the others' weights are below 2^-100)


@gpu
def test_a_cache_of_8_bits_past_32_bits(rk):
    """Five KV heads of 2^23 rows of 8 bits, new rows that fill a block and begin the next."""
    n, cap, block, H, T = (1 << 23) + 57, (1 << 23) + 64, 64, 5, 80
    geom = rk.Geom(1, H, H, 128, SCALE)
    cache = rk.Kv8.empty(geom, cap, block, torch.int8)
    g = torch.Generator().manual_seed(10)
    k, v = (torch.randn(1, T, H, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    sl = i32([n])
    rk.rk_rope_append_q8(geom, None, k.cuda(), v.cuda(), None, cache, sl, None)
    rows = []                                                                    # [key, value][head]: the last 64 + 57 rows
    for x in (k, v):
        rows.append([])
        for h in range(H):
            held = o.Cache8(block, "int8")
            for r in [np.zeros(128, np.uint16)] * (block - (T - 57)) + list(gen.bf16_bits(x)[0, :, h]):      # (the tail was empty: zeros)
                held.append(r)
            rows[-1].append(held.rows())
    at = n - (block + 57)
    pick = np.array([block - (T - 57), 63, 64, 64 + 56])                         # in both blocks
    sK, sV = (torch.zeros(1, H, 5, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rk.rk_gather_small_kv_q8(geom, cache, i32([[[int(at + x) for x in (*pick, pick[0])]] * H]), 5, sK, sV, sl)
    torch.cuda.synchronize()
    for h in range(H):
        for got, x in ((sK, rows[0][h]), (sV, rows[1][h])):
            assert np.array_equal(gen.bf16_bits(got.cpu())[0, h, :4], o.f64_to_bf16_bits(x[pick])) and torch.equal(got[0, h, 0], got[0, h, 4])      # (the same row twice)
    ws = rk.Workspace(geom, cap, 1)
    w, out, lse = torch.zeros(1, H, cap, device="cuda"), torch.zeros(1, H, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(1, H, device="cuda")
    for j in (63, 64 + 56):                                                      # a row of 8 bits, a row of the tail
        q = torch.from_numpy(40 * np.stack([rows[0][h][j] for h in range(H)])).to(torch.bfloat16)[None].cuda()
        rk.rk_full_attn_q8(geom, q, cache, sl, cap, out, weights=w, lse=lse, workspace=ws)
        torch.cuda.synchronize()
        for h in range(H):
            # scores of several hundred, fp32's steps there 2^-15: the row has all the weight to within 2^-10
            assert int(w[0, h, :n].argmax()) == at + j and abs(float(w[0, h, at + j]) - 1) <= 2.0 ** -10
            # one rounding of a row whose weight is 1 to 2^-17
            want = rows[1][h][j]
            assert (np.abs(out[0, h].double().cpu().numpy() - want) <= (2.0 ** -8 + 2.0 ** -16) * np.abs(want) + 2.0 ** -16 * np.abs(rows[1][h]).max()).all()


@gpu
def test_two_servers_at_once(rk):
    """The whole chain on two streams at the same time, each with its own cache and scratch, has the results of one after the other."""
    B, Hq, H, cap, T, k = 2, 8, 2, 2048, 40, 64
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator(device="cuda").manual_seed(8)
    sides = []
    for _ in range(2):
        w = torch.randn(B, T, Hq + 2 * H, 128, generator=g, device="cuda").to(torch.bfloat16)
        K, V = (torch.randn(B, H, cap, 128, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        sides.append((w, K, V))
    rope = rk.Rope(rk.rope_table(cap, 128))

    def chain(side):
        w, K, V = side[0], side[1].clone(), side[2].clone()
        cache, ws, pws = rk.Kv8.empty(geom, cap, 32, torch.int8), rk.Workspace(geom, cap, k), rk.PromptWorkspace(geom, T, cap)
        old = i32([2000, 1500])
        rk.rk_rope_append_q8(geom, None, K[:, :, :2000].transpose(1, 2).contiguous(), V[:, :, :2000].transpose(1, 2).contiguous(), None, cache, old, None, new_lens=old)
        got = []
        for r in range(6):
            sl = old + r + T
            qo, out = torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda")
            rk.rk_rope_append(geom, w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:], rope, K, V, sl, qo)
            rk.rk_prompt_attn(geom, qo, K, V, sl, cap, out, workspace=pws)
            q1 = qo[:, r].contiguous()
            rk.rk_rope_append_q8(geom, None, w[:, r:r + 1, Hq:Hq + H], w[:, r:r + 1, Hq + H:], rope, cache, old + r + 1, None)
            o1, wt, idx = torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hq, cap, device="cuda"), torch.zeros(B, H, k, dtype=torch.int32, device="cuda")
            rk.rk_full_attn_q8(geom, q1, cache, old + r + 1, cap, o1, weights=wt, workspace=ws)
            rk.rk_topk_select(geom, wt, old + r + 1, cap, k, 7, idx, workspace=ws)
            sK, sV = torch.zeros(2, B, H, k, 128, dtype=torch.bfloat16, device="cuda")
            rk.rk_gather_small_kv_q8(geom, cache, idx, k, sK, sV, old + r + 1)
            got += [qo, out, o1, wt, idx, sK, sV]
        return got + [K, V, cache.k.view(torch.uint8), cache.k_scale, cache.v_tail]
    one = [chain(x) for x in sides]
    torch.cuda.synchronize()
    streams, both = [torch.cuda.Stream() for _ in range(2)], []
    for s_, x in zip(streams, sides):
        with torch.cuda.stream(s_):
            both.append(chain(x))
    torch.cuda.synchronize()
    for a, b in zip(one, both):
        for x, y in zip(a, b):
            assert torch.equal(x, y)


@gpu
@pytest.mark.parametrize("eight", [False, True])
def test_appended_rows_at_the_edges(rk, eight):
    """One token's rows for all sequences (a batch stride of 0), counts outside 0 .. n_new, sequences that the predicate leaves alone, lengths below the count."""
    B, Hq, H, T, cap = 4, 4, 2, 5, 64
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    g = torch.Generator().manual_seed(19)
    w = torch.randn(1, T, Hq + 2 * H, 128, generator=g).to(torch.bfloat16).cuda()
    wide = w.expand(B, T, Hq + 2 * H, 128)
    rope = rk.Rope(rk.rope_table(cap, 64))
    lens, new, pred = [5, 40, 3, 50], [99, -3, 5, 2], [1, 1, 1, 0]

    def run(rows, into):
        qo = torch.full((B, T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
        args = (geom, rows[:, :, :Hq], rows[:, :, Hq:Hq + H], rows[:, :, Hq + H:], rope)
        kw = dict(new_lens=i32(new), pred=i32(pred), pred_val=1)
        if eight:
            rk.rk_rope_append_q8(*args, into, i32(lens), qo, **kw)
        else:
            rk.rk_rope_append(*args, *into, i32(lens), qo, **kw)
        torch.cuda.synchronize()
        return qo

    def room():
        if eight:
            return rk.Kv8.empty(geom, cap, 16)
        return [torch.full((B, H, cap, 128), 3.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    a, b = room(), room()
    qa, qb = run(wide, a), run(wide.contiguous(), b)
    held = lambda x: [getattr(x, n).view(torch.uint8) for n in ("k", "v", "k_scale", "v_scale", "k_tail", "v_tail")] if eight else x  # noqa: E731
    assert torch.equal(qa.view(torch.int16), qb.view(torch.int16)) and all(torch.equal(x, y) for x, y in zip(held(a), held(b)))
    assert (qa[1] == 7).all() and (qa[3] == 7).all()                             # none; left alone
    # three rows of a sequence of 3 with five new ones: entries 2 .. 4; the first two lie before the cache, and their position is in no table
    assert qa[2, :2, :, :64].isnan().all() and torch.equal(qa[2, :2, :, 64:], w[0, :2, :Hq, 64:].expand(2, Hq, 64)) and qa[2, 2:].isfinite().all()
    if eight:
        assert not a.k_tail[1].any() and not a.k_tail[3].any() and a.k_tail[2, :, :3].isfinite().all() and not a.k_tail[2, :, 3:].any()
        assert torch.equal(a.v_tail[2, :, :3], w[0, 2:5, Hq + H:].transpose(0, 1)) and torch.equal(a.v_tail[0, :, :5], w[0, :, Hq + H:].transpose(0, 1))
    else:
        assert (a[1][1] == 3).all() and (a[1][3] == 3).all() and torch.equal(a[1][2, :, :3], w[0, 2:5, Hq + H:].transpose(0, 1)) and (a[1][2, :, 3:] == 3).all()
        assert torch.equal(a[1][0, :, :5], w[0, :, Hq + H:].transpose(0, 1))


FORMS = {"plain": "", "strided": "", "stream": "", "parameter": "", "subclass": "append append8 full8 gather8 prompt", "numpy_int": "full8 gather8 prompt",
         "wrong_shape": "append append8 full8 prompt", "wrong_type": "append append8 full8 prompt", "other_geometry": "append8 full8 gather8", "int_cap": "prompt"}


class _Sub(torch.Tensor):
    pass


@gpu
@pytest.mark.parametrize("form", list(FORMS))
def test_calls_marshalled_in_cpp_take_what_python_takes(rk, form, monkeypatch):
    """The same results, or the same exception, through the C++ checks as through those of binding.py alone."""
    B, G, H, n, k, T = 2, 4, 2, 200, 32, 9
    Hq = G * H
    g = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(torch.bfloat16)  # noqa: E731
    geom = rk.Geom(B, Hq, H, 128, SCALE)
    w = rnd(B, T, Hq + 2 * H, 128)
    q, nk, nv = w[:, :, :Hq], w[:, :, Hq:Hq + H], w[:, :, Hq + H:]
    q1 = rnd(B, Hq, 128)
    K0, V0 = rnd(B, H, 208, 128), rnd(B, H, 208, 128)
    rope = rk.Rope(rk.rope_table(256, 64), interleaved=True)
    idx = torch.randint(0, n - 9, (B, H, k), generator=g, device="cuda", dtype=torch.int32)
    n_int, n_sel, cap, stream, geom8 = n, k, 5.0, None, geom
    if form == "strided":
        K0, V0 = rnd(B, H + 2, 215, 128)[:, 1:-1, :208], rnd(B, H + 2, 215, 128)[:, 1:-1, :208]
    elif form == "stream":
        stream = torch.cuda.Stream()
    elif form == "parameter":
        q, q1 = torch.nn.Parameter(q, requires_grad=False), torch.nn.Parameter(q1, requires_grad=False)
    elif form == "subclass":
        q, q1, idx = q.as_subclass(_Sub), q1.as_subclass(_Sub), idx.as_subclass(_Sub)
    elif form == "numpy_int":
        n_int, n_sel = np.int64(n), np.int64(k)
    elif form == "wrong_shape":
        q, q1 = q[:, :, 1:], q1[:, 1:].contiguous()
    elif form == "wrong_type":
        q, q1 = q.float(), q1.float()
    elif form == "other_geometry":
        geom8 = rk.Geom(B, Hq, H, 128, 2 * SCALE)                                # (of the same sizes: taken, but by binding.py)
    elif form == "int_cap":
        cap = 5

    def run():
        ws, pws = rk.Workspace(geom, 208, k), rk.PromptWorkspace(geom, T, 208)
        lens, new, pred = i32([n, n - 7]), i32([T, 3]), i32([1, 1])
        K, V = K0.clone().contiguous(), V0.clone().contiguous()
        if form == "strided":
            K, V = (torch.zeros(B, H + 2, 215, 128, dtype=torch.bfloat16, device="cuda")[:, 1:-1, :208].copy_(x) for x in (K0, V0))
        cache = rk.Kv8.empty(geom8, 208, 16)
        rk.rk_rope_append_q8(geom8, None, K0[:, :, :n].transpose(1, 2).contiguous(), V0[:, :, :n].transpose(1, 2).contiguous(), None, cache, lens - 9, None)
        qo = [torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda") for _ in range(3)]
        o1, lse1, wt = torch.zeros(B, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(B, Hq, device="cuda"), torch.zeros(B, Hq, 208, device="cuda")
        lse = torch.zeros(B, T, Hq, device="cuda")
        sK, sV = torch.zeros(2, B, H, k, 128, dtype=torch.bfloat16, device="cuda")
        tail = i32([-1, -1])
        if stream is not None:
            stream.wait_stream(torch.cuda.current_stream())
        res = {}
        for name, call in (
                ("append", lambda: rk.rk_rope_append(geom, q, nk, nv, rope, K, V, lens, qo[0], new_lens=new, pred=pred, pred_val=1, stream=stream)),
                ("append8", lambda: rk.rk_rope_append_q8(geom, q, nk, nv, rope, cache, lens, qo[1], new_lens=i32([9, 2]), stream=stream)),
                ("full8", lambda: rk.rk_full_attn_q8(geom, q1, cache, lens, n_int, o1, weights=wt, lse=lse1, workspace=ws, stream=stream)),
                ("gather8", lambda: rk.rk_gather_small_kv_q8(geom, cache, idx, n_sel, sK, sV, lens, tail_start=tail, stream=stream)),
                ("prompt", lambda: rk.rk_prompt_attn(geom, q, K, V, lens, n_int, qo[2], new_lens=new, cap=cap, lse=lse, workspace=pws, stream=stream))):
            try:
                call()
                res[name] = None
            except (ValueError, TypeError) as e:
                res[name] = str(e)
        torch.cuda.synchronize()
        return res, [K, V, *qo, o1, lse1, wt, lse, sK, sV, tail, cache.k.view(torch.uint8), cache.k_scale, cache.v_tail]

    taken = []

    def watched(call):
        def f(*a):
            taken.append(call(*a) is not None)
            return 0 if taken[-1] else None
        return f
    names = ("rk_rope_append", "rk_rope_append_q8", "rk_full_attn_q8", "rk_gather_small_kv_q8", "rk_prompt_attn")
    native = rk.binding._native
    monkeypatch.setattr(rk.binding, "_native", type("watched", (), {x: staticmethod(watched(getattr(native, x))) for x in names}))
    by_cpp = run()
    monkeypatch.setattr(rk.binding, "_native", type("none", (), {x: staticmethod(lambda *a: None) for x in names}))
    by_python = run()
    assert by_cpp[0] == by_python[0], (by_cpp[0], by_python[0])
    taken = taken[1:]                                                            # (the call that fills the cache)
    assert [x for x, t in zip(by_cpp[0], taken) if not t] == FORMS[form].split() and len(taken) == 5
    assert any(by_cpp[0].values()) == (form in ("wrong_shape", "wrong_type"))
    for a, b in zip(by_cpp[1], by_python[1]):
        assert torch.equal(a, b)
