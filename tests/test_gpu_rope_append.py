"""rk_rope_table, rk_rope_append, rk_rope_append_q8: refusals (no GPU needed), and against oracle/new_tokens.py."""
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


# ---- refusals ----

def test_refusals_before_any_launch(rk):
    from paper_2411_05787_amd.binding import _Geom, _Kv, _Kv8, _NewRows, _Rope, _RopeScaling
    g, f = _Geom(2, 32, 8, 128, 0.1), 0x10000
    kv = _Kv(f, f, 8 * 64 * 128, 64 * 128, 64)

    def rows(q=f, k=f, v=f, st=6144, n=3):
        return _NewRows(q, k, v, 3 * st, st, 3 * st, st, 3 * st, st, n)

    def append(geom=g, r=rows(), rope=_Rope(f, 64, 128, 0), cache=kv, sl=f, qo=f):
        return rk.lib.rk_rope_append(C.byref(geom), C.byref(r), None if rope is None else C.byref(rope), None, cache, sl, None, qo, None, 0, None)

    assert append(geom=_Geom(2, 32, 8, 64, 0.1)) == -2
    assert append(r=rows(k=None)) == -1 and append(r=rows(v=None)) == -1 and append(sl=None) == -1
    assert append(r=rows(n=0)) == -1
    assert append(r=rows(q=None)) == -1 and append(qo=None) == -1              # q and q_out go together
    assert append(rope=None) == -1                                             # a copy of q is not made
    assert append(r=rows(k=f + 2)) == -1 and append(qo=f + 8) == -1            # 16-byte alignment
    assert append(r=rows(st=6140)) == -1 and append(r=rows(st=-8)) == -1
    assert append(rope=_Rope(None, 64, 128, 0)) == -1 and append(rope=_Rope(f, 0, 128, 0)) == -1
    assert append(rope=_Rope(f, 64, 120, 0)) == -2 and append(rope=_Rope(f, 64, 144, 0)) == -2 and append(rope=_Rope(f, 64, 0, 0)) == -2
    assert append(cache=_Kv(f, None, 0, 0, 64)) == -1
    assert append(r=rows(n=2 ** 31 - 1)) == -2                                 # more rows than a grid takes

    def c8(k=f, cap=64, block=32, fmt=0, tail=f, sh=64 * 128, scale=f):
        return _Kv8(k, f, scale, f, tail, f, 8 * 64 * 128, sh, cap, block, fmt)

    def append8(c=c8(), **kw):
        return rk.lib.rk_rope_append_q8(C.byref(g), C.byref(kw.get("r", rows())), C.byref(_Rope(f, 64, 128, 0)), None, C.byref(c), f, None, f, None, 0, None)

    assert append8(c8(fmt=2)) == -2 and append8(c8(block=8)) == -2 and append8(c8(block=48)) == -2 and append8(c8(block=256, cap=256)) == -2
    assert append8(c8(cap=72)) == -1 and append8(c8(cap=0)) == -1 and append8(c8(k=None)) == -1 and append8(c8(tail=None)) == -1
    assert append8(c8(k=f + 8)) == -1 and append8(c8(tail=f + 8)) == -1 and append8(c8(scale=f + 2)) == -1
    assert append8(c8(sh=64 * 128 + 8)) == -1 and append8(c8(sh=2 ** 31)) == -2
    assert append8(r=rows(k=None)) == -1

    def table(t=f, n=8, rot=128, s=_RopeScaling(1e4, 1, 0, 0, 0, 1)):
        return rk.lib.rk_rope_table(t, n, rot, C.byref(s), None)

    assert table(t=None) == -1 and table(n=0) == -1 and table(rot=100) == -2
    assert table(s=_RopeScaling(0, 1, 0, 0, 0, 1)) == -1 and table(s=_RopeScaling(1e4, 0, 0, 0, 0, 1)) == -1
    assert table(s=_RopeScaling(1e4, 8, 4, 4, 8192, 1)) == -1 and table(s=_RopeScaling(1e4, 1, 0, 0, 0, math.nan)) == -1


def test_binding_refuses(rk):
    g = rk.Geom(1, 4, 2, 128, 0.1)
    x = torch.zeros(1, 3, 4, 128, dtype=torch.bfloat16)
    with pytest.raises(ValueError):
        rk.Rope(torch.zeros(8, 128))                                           # not in GPU memory
    with pytest.raises(ValueError):
        rk.rk_rope_append(g, x, x[:, :, :2], x[:, :, :2], None, x, x, torch.zeros(1, dtype=torch.int32), x)
    with pytest.raises(ValueError):
        rk.Kv8(g, *(torch.zeros(1, 2, 32, 128, dtype=torch.int8) for _ in range(2)), *(torch.zeros(1, 2, 1) for _ in range(2)),
               *(torch.zeros(1, 2, 32, 128, dtype=torch.bfloat16) for _ in range(2)))


# ---- the table ----

@gpu
@pytest.mark.parametrize("kw", [dict(), dict(factor=4.0), dict(base=500000.0, factor=8.0, low_turns=1.0, high_turns=4.0, original_len=8192),
                                dict(base=1e6, factor=16.0, low_turns=1.0, high_turns=32.0, original_len=4096, amplitude=1.2772588722239781)])
@pytest.mark.parametrize("rot", [128, 48])
def test_table(rk, kw, rot):
    say("table", kw, rot)
    n = 131072 if rot == 48 else 5000
    t = rk.rope_table(n, rot, **kw).cpu().double().numpy()
    args = {k: v for k, v in kw.items() if k != "amplitude"}
    f = o.rope_frequencies(rot, args.pop("base", 10000.0), **args)
    at = np.unique(np.concatenate([np.arange(50), np.geomspace(50, n - 1, 200).astype(int)]))
    a, amp = at[:, None] * f, kw.get("amplitude", 1.0)
    # one rounding to fp32, and angles of up to 2^17 in fp64 (frequencies from two implementations of pow): 2^-24 relative and 2^17 * 2^-51
    want = np.concatenate([amp * np.cos(a), amp * np.sin(a)], axis=1)
    assert (np.abs(t[at] - want) <= 2.0 ** -24 * np.abs(want) + amp * 2.0 ** -34).all()


# ---- into the bf16 cache ----

def bits(t):
    return gen.bf16_bits(t)


def close_turn(got_bits, x, cos, sin, inter, what):
    """fp32 products and sums, one rounding to bf16: half a step (2^-8 relative) and three roundings of 2^-24 of the terms."""
    want = o.rope_turn(x, cos, sin, inter)
    size = np.abs(o.rope_turn(np.abs(x), np.abs(cos), -np.abs(sin), inter)) + np.abs(o.rope_turn(np.abs(x), np.abs(cos), np.abs(sin), inter))
    got = o.bf16_bits_to_f64(got_bits)
    assert (np.abs(got - want) <= 2.0 ** -8 * np.abs(want) + 3 * 2.0 ** -24 * size).all(), what


CASES = [
    # B, Hq, Hkv, n_new, lens, new_lens, rot, interleaved, capacity
    ("step", 1, 32, 8, 1, [17], None, 128, False, 64),
    ("first_token", 2, 28, 4, 1, [1, 64], None, 128, True, 64),
    ("half_of_the_head", 1, 8, 8, 5, [40], None, 64, False, 48),
    ("sixteen_dims", 1, 5, 1, 3, [3], None, 16, True, 16),
    ("ragged", 3, 20, 4, 33, [33, 200, 77], [33, 0, 12], 96, False, 208),
    ("ragged_interleaved", 2, 64, 8, 70, [70, 300], [70, 1], 112, True, 304),
    ("beyond_the_cache", 2, 4, 2, 9, [20, 5], [9, 9], 128, False, 16),          # rows from 16 on, and before 0, are not there
    ("many_rows", 2, 32, 8, 1500, [1500, 1400], [1500, 1399], 128, False, 1504),
]


def one(rk, case, seed=0, strided=True):
    name, B, Hq, H, T, lens, new, rot, inter, cap = case
    g = torch.Generator().manual_seed(seed)
    w = torch.randn(B, T, Hq + 2 * H, 128, generator=g).to(torch.bfloat16)
    K0, V0 = (torch.randn(B, H, cap, 128, generator=g).to(torch.bfloat16) for _ in range(2))
    geom = rk.Geom(B, Hq, H, 128, 0.1)
    table = rk.rope_table(max(lens) + T, rot)
    wd = w.cuda()
    q, k, v = wd[:, :, :Hq], wd[:, :, Hq:Hq + H], wd[:, :, Hq + H:]
    if not strided:
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    sl = torch.tensor(lens, dtype=torch.int32, device="cuda")
    nl = None if new is None else torch.tensor(new, dtype=torch.int32, device="cuda")
    return geom, w, K0, V0, rk.Rope(table, inter), q, k, v, sl, nl, table.cpu().double().numpy()


@gpu
@pytest.mark.parametrize("case", CASES, ids=[c[0] for c in CASES])
def test_append(rk, case):
    name, B, Hq, H, T, lens, new, rot, inter, cap = case
    say("append", name)
    geom, w, K0, V0, rope, q, k, v, sl, nl, table = one(rk, case)
    K, V = K0.cuda(), V0.cuda()
    qo = torch.full((B, T, Hq, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    rk.rk_rope_append(geom, q, k, v, rope, K, V, sl, qo, new_lens=nl)
    torch.cuda.synchronize()
    x = o.bf16_bits_to_f64(bits(w))
    wantK, wantV, Kb, Vb, qb = bits(K0).copy(), bits(V0).copy(), bits(K), bits(V), bits(qo)
    for b in range(B):
        n = T if new is None else new[b]
        start = lens[b] - n
        at = np.arange(start, lens[b])
        pos = at[:, None]
        ok = at >= 0
        cos, sin = (table[np.clip(at, 0, None)][:, None, s] for s in (slice(0, rot // 2), slice(rot // 2, rot)))
        if n:
            close_turn(qb[b, :n][ok], x[b, :n, :Hq][ok], cos[ok], sin[ok], inter, name + " q")
            assert np.isnan(o.bf16_bits_to_f64(qb[b, :n][~ok])[..., :rot]).all()       # a position before 0
        assert (o.bf16_bits_to_f64(qb[b, n:]) == 7.0).all()
        for i, r in enumerate(at):
            if not 0 <= r < cap:
                continue
            close_turn(Kb[b, :, r], x[b, i, Hq:Hq + H], cos[i], sin[i], inter, name + " k")
            wantK[b, :, r] = Kb[b, :, r]
            wantV[b, :, r] = bits(w)[b, i, Hq + H:]
    assert (Kb == wantK).all() and (Vb == wantV).all()                          # and nothing else was touched


@gpu
def test_append_in_place_positions_predicate(rk):
    case = ("x", 3, 12, 4, 21, [21, 40, 33], [21, 5, 17], 128, False, 48)
    geom, w, K0, V0, rope, q, k, v, sl, nl, _ = one(rk, case, strided=False)
    K, V, qo = K0.cuda(), V0.cuda(), torch.zeros_like(q)
    rk.rk_rope_append(geom, q, k, v, rope, K, V, sl, qo, new_lens=nl)
    K2, V2, q2 = K0.cuda(), V0.cuda(), q.clone()
    rk.rk_rope_append(geom, q2, k, v, rope, K2, V2, sl, q2, new_lens=nl)        # q_out is q
    assert torch.equal(K, K2) and torch.equal(V, V2)
    for b, n in enumerate(case[6]):
        assert torch.equal(qo[b, :n], q2[b, :n]) and torch.equal(q2[b, n:], q[b, n:])
    # explicit positions: those of the rows give the same bits, shifted ones another turn; out of the table: NaN in the turned dims
    pos = (sl - nl)[:, None] + torch.arange(21, device="cuda", dtype=torch.int32)
    K3, V3, q3 = K0.cuda(), V0.cuda(), torch.zeros_like(q)
    rk.rk_rope_append(geom, q, k, v, rope, K3, V3, sl, q3, new_lens=nl, positions=pos.int().contiguous())
    assert torch.equal(K, K3) and torch.equal(qo, q3)
    far = torch.full((3, 21), 10 ** 6, dtype=torch.int32, device="cuda")
    rk.rk_rope_append(geom, q, k, v, rope, K3, V3, sl, q3, new_lens=nl, positions=far)
    assert q3[0].isnan().all() and torch.equal(V, V3)
    # only the predicate's sequences; no q; nothing turned
    K4, V4 = K0.cuda(), V0.cuda()
    pred = torch.tensor([1, 0, 1], dtype=torch.int32, device="cuda")
    rk.rk_rope_append(geom, None, k, v, rope, K4, V4, sl, None, new_lens=nl, pred=pred, pred_val=1)
    assert torch.equal(K4[0], K[0]) and torch.equal(K4[1], K0[1].cuda()) and torch.equal(V4[2], V[2])
    rk.rk_rope_append(geom, None, k, v, None, K4, V4, sl, None, new_lens=nl)
    assert torch.equal(K4[0, :, :21], k[0].transpose(0, 1)) and torch.equal(V4, V)


# ---- into the cache of 8 bits ----

Q8_CASES = [
    # B, Hkv, block, format, pieces: new tokens of each sequence, call by call (0: none)
    ("steps", 1, 2, 16, "e4m3", [[1]] * 35),
    ("steps_int8", 2, 1, 16, "int8", [[1, 1]] * 18),
    ("prompt", 1, 4, 32, "e4m3", [[100]]),
    ("pieces", 3, 2, 32, "int8", [[50, 1, 0], [13, 31, 32], [1, 1, 1], [70, 0, 63]]),
    ("pieces_128", 2, 2, 128, "e4m3", [[127, 128], [1, 129], [300, 1]]),
    ("pieces_64", 2, 3, 64, "int8", [[63, 65], [2, 62], [64, 64], [129, 128]]),
]


@gpu
@pytest.mark.parametrize("gain", [1.0, 1e-30, 3e30])
@pytest.mark.parametrize("case", Q8_CASES, ids=[c[0] for c in Q8_CASES])
def test_append_q8_bits(rk, case, gain):
    """Bit for bit the oracle's cache, whatever the pieces."""
    name, B, H, blk, fmt, pieces = case
    say("append_q8", name, gain)
    total = np.array(pieces).sum(axis=0)
    cap = (int(total.max()) + blk - 1) // blk * blk
    g = torch.Generator().manual_seed(5)
    rows = {n: (torch.randn(B, int(total.max()), H, 128, generator=g) * torch.exp(torch.randn(B, int(total.max()), 1, 1, generator=g)) * gain).to(torch.bfloat16)
            for n in "kv"}
    rows["v"][0, 3] = 0                                                          # a row of zeros; a block of them with the next line
    if blk == 16:
        rows["k"][0, 16:32] = 0
    dtype = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    geom = rk.Geom(B, H, H, 128, 0.1)
    cache = rk.Kv8.empty(geom, cap, blk, dtype)
    have = np.zeros(B, dtype=int)
    for new in pieces:
        T = max(new)
        part = {n: torch.zeros(B, T, H, 128, dtype=torch.bfloat16) for n in "kv"}
        for b in range(B):
            for n in "kv":
                part[n][b, :new[b]] = rows[n][b, have[b]:have[b] + new[b]]
        have += np.array(new)
        rk.rk_rope_append_q8(geom, None, part["k"].cuda(), part["v"].cuda(), None, cache, torch.tensor(have, dtype=torch.int32, device="cuda"), None,
                             new_lens=torch.tensor(new, dtype=torch.int32, device="cuda"))
    torch.cuda.synchronize()
    for n in "kv":
        x8 = getattr(cache, n).view(torch.uint8).cpu().view(dtype).double().numpy()
        scales, tail = getattr(cache, n + "_scale").cpu().double().numpy(), bits(getattr(cache, n + "_tail"))
        for b in range(B):
            for h in range(H):
                want = o.Cache8(blk, fmt)
                for r in range(total[b]):
                    want.append(bits(rows[n])[b, r, h])
                for i, (v, s) in enumerate(zip(want.values, want.scales)):
                    assert scales[b, h, i] == s, (n, b, h, i)
                    assert (x8[b, h, i * blk:(i + 1) * blk] == v).all(), (n, b, h, i)
                full = total[b] // blk
                assert (scales[b, h, full:] == 0).all() and (x8[b, h, full * blk:] == 0).all()
                assert (bits(rows[n])[b, full * blk:total[b], h] == tail[b, h, :total[b] - full * blk]).all()


@gpu
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_append_q8_every_value_and_non_finite(rk, fmt):
    """Every finite bf16 within a block's range of its largest, ties among them; a block with an infinity or a NaN."""
    dtype = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    allb = torch.arange(65536, dtype=torch.int32).to(torch.int16).view(torch.bfloat16)
    most = 448.0 if fmt == "e4m3" else 127.0
    fine = allb[torch.isfinite(allb) & (allb.abs() <= most)]
    blk, D = 128, 128
    n = (len(fine) + blk * D - 2) // (blk * D - 1)
    x = torch.zeros(n, blk * D, dtype=torch.bfloat16)
    x[:, 0] = most                                                               # every block's scale is 1
    for i in range(n):
        part = fine[i * (blk * D - 1):(i + 1) * (blk * D - 1)]
        x[i, 1:1 + len(part)] = part
    geom = rk.Geom(1, 1, 1, 128, 0.1)
    cache = rk.Kv8.empty(geom, (n + 2) * blk, blk, dtype)
    rows = torch.cat([x.view(1, n * blk, 1, D), torch.zeros(1, 2 * blk, 1, D, dtype=torch.bfloat16)], dim=1)
    rows[0, n * blk + 5, 0, 7] = float("inf")
    rows[0, (n + 1) * blk + 5, 0, 7] = float("nan")
    rk.rk_rope_append_q8(geom, None, rows.cuda(), rows.cuda(), None, cache, torch.tensor([(n + 2) * blk], dtype=torch.int32, device="cuda"), None)
    torch.cuda.synchronize()
    for t, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)):
        assert (s[0, 0, :n] == 1).all() and s[0, 0, n:].isnan().all()
        got = t.view(torch.uint8).cpu().view(dtype).double().numpy()[0, 0]
        assert (got[:n * blk] == o.nearest_value(x.double().numpy().reshape(n * blk, D), fmt)).all() and (got[n * blk:] == 0).all()


@gpu
def test_append_q8_turns_as_the_bf16_append_does(rk):
    """q_out and the turned keys of both appends are the same bits; rows beyond the capacity are dropped, the predicate holds."""
    B, Hq, H, T, blk = 2, 28, 4, 150, 32
    case = ("x", B, Hq, H, T, [150, 190], [150, 130], 96, True, 192)
    geom, w, K0, V0, rope, q, k, v, sl, nl, _ = one(rk, case)
    K, V, qo = K0.cuda(), V0.cuda(), torch.zeros(B, T, Hq, 128, dtype=torch.bfloat16, device="cuda")
    rk.rk_rope_append(geom, q, k, v, rope, K, V, sl, qo, new_lens=nl)
    cache, q8 = rk.Kv8.empty(geom, 192, blk, torch.int8), torch.zeros_like(qo)
    rk.rk_rope_append_q8(geom, q, k, v, rope, cache, sl, q8, new_lens=nl)
    assert torch.equal(qo, q8)
    for b, (n, new) in enumerate(((150, 150), (190, 130))):
        for t, tail, full, scale in ((K, cache.k_tail, cache.k, cache.k_scale), (V, cache.v_tail, cache.v, cache.v_scale)):
            last = n // blk * blk
            assert torch.equal(tail[b, :, :n - last], t[b, :, last:n])
            # whole blocks of new rows: half a step of the format at most
            lo = (n - new + blk - 1) // blk * blk
            got = full[b, :, lo:last].double() * scale[b, :, lo // blk:last // blk].double().repeat_interleave(blk, dim=1)[..., None]
            assert ((got - t[b, :, lo:last].double()).abs() <= 0.5 * scale[b, :, lo // blk:last // blk].double().repeat_interleave(blk, dim=1)[..., None]).all()
    short, q9 = rk.Kv8.empty(geom, 160, blk, torch.int8), torch.zeros_like(qo)
    pred = torch.tensor([0, 1], dtype=torch.int32, device="cuda")
    rk.rk_rope_append_q8(geom, q, k, v, rope, short, sl, q9, new_lens=nl, pred=pred, pred_val=1)
    assert torch.equal(short.k[1], cache.k[1, :, :160]) and torch.equal(short.v_scale[1], cache.v_scale[1, :, :5])
    assert (short.k_tail == 0).all() and (short.k[0] == 0).all() and torch.equal(q9[1], qo[1]) and (q9[0] == 0).all()
