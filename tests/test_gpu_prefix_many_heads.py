"""rk_prefix_attn where all query rows of a KV head together are columns (16 at most) and (sequence, KV head) pairs are more than the compute units: plain
multi-head models with a few sequences.  Against oracle/paged.py; the scratch holds zeros before each call, so that a pair that nobody went over shows."""
import pytest
import torch

from test_gpu_paged_attn import Inputs, i32, rk, say  # noqa: F401

pytestmark = pytest.mark.gpu

CASES = {
    "sixteen_of_32": dict(B=16, Hq=32, H=32, T=1, lens=[90 + 7 * i for i in range(16)], new=None, page=16, prefix=80),
    "nine_of_29": dict(B=9, Hq=29, H=29, T=1, lens=[200 - 11 * i for i in range(9)], new=None, page=32, prefix=70),
    "five_of_64": dict(B=5, Hq=64, H=64, T=1, lens=[130, 129, 0, 140, 300], new=[1, 0, 0, 1, 1], page=16, prefix=128),
    "drafted": dict(B=3, Hq=100, H=100, T=5, lens=[150, 101, 260], new=[5, 1, 4], page=64, prefix=100),
    "two_heads_to_a_group": dict(B=4, Hq=140, H=70, T=2, lens=[75, 90, 61, 120], new=None, page=16, prefix=60, cap=5.0, slopes=True),
    "window": dict(B=14, Hq=20, H=20, T=1, lens=[100 + 5 * i for i in range(14)], new=None, page=16, prefix=90, masks="window"),
    "missing": dict(B=10, Hq=27, H=27, T=1, lens=[140 + 3 * i for i in range(10)], new=None, page=16, prefix=96, missing=2),
    "at_the_units": dict(B=8, Hq=64, H=32, T=1, lens=[100 + i for i in range(8)], new=None, page=16, prefix=64),
    "split_own": dict(B=1, Hq=257, H=257, T=1, lens=[700], new=None, page=16, prefix=40),
}


@pytest.mark.parametrize("name", list(CASES))
def test_prefix(rk, name):  # noqa: F811
    say("prefix, many heads", name)
    x = Inputs(**CASES[name])
    geom, pages, q, table, lens, args = x.device(rk)
    own = max(1, max(x.lens) - x.prefix)
    ws = rk.PrefixWorkspace(geom, x.T, x.prefix, own)
    pt, pl = i32(x.prefix_table), i32([x.prefix])
    assert x.B * x.T * x.G <= 16
    outs = []
    for _ in range(2):
        ws.buf.zero_()
        out, lse = x.blank()
        rk.rk_prefix_attn(geom, q, pages, pt, pl, x.prefix, table, lens, own, out, lse=lse, workspace=ws, **args)
        torch.cuda.synchronize()
        outs.append((out, lse))
    x.check(*outs[0], True, name)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_captured_beside_eager_calls(rk):  # noqa: F811
    """Replayed with other lengths, eager calls with scratch of their own between the replays."""
    x = Inputs(B=11, Hq=30, H=30, T=1, lens=[200] * 11, new=None, page=16, prefix=64)
    geom, pages, q, table, lens, args = x.device(rk)
    ws = [rk.PrefixWorkspace(geom, 1, 64, 200) for _ in range(2)]
    pt, pl = i32(x.prefix_table), i32([64])
    held, eager = x.blank(), x.blank()

    def run(to, w):
        rk.rk_prefix_attn(geom, q, pages, pt, pl, 64, table, lens, 200, to[0], lse=to[1], workspace=w, **args)
    run(held, ws[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(held, ws[0])
    for n in (200, 65, 130, 64, 3, 199):
        lens.copy_(i32([max(n - i, 0) for i in range(11)]))
        ws[0].buf.zero_()
        graph.replay()
        run(eager, ws[1])
        torch.cuda.synchronize()
        assert torch.equal(held[0], eager[0]) and torch.equal(held[1], eager[1]), n
