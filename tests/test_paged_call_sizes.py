"""Sizes that the calls over pages take, by what they launch (no GPU needed): a launch has fewer than 2^32 threads along its first axis, and what would not
be launched bounds nothing."""
import ctypes as C

import pytest

FAR = 0x10000                                                                    # never read: without a GPU no launch begins, and a refusal comes before it
UNSUPPORTED = -2


@pytest.fixture(scope="module")
def calls():
    """The status of a call of a shape with made-up addresses: UNSUPPORTED, or another one of a launch that no GPU is there for."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("calls with made-up addresses are for machines without a GPU")
    import paper_2411_05787_amd as rk
    from paper_2411_05787_amd.binding import _Geom, _Kv, _Pages
    lib = rk.lib

    class Calls:
        def __init__(self, B, Hq, H, T, rows, k=8, page=32):
            self.g, self.gp = _Geom(B, Hq, H, 128, 0.1), None
            self.kv = _Kv(FAR, FAR, H * rows * 128, rows * 128, rows)
            self.pages = _Pages(FAR, FAR, None, None, H * page * 128, page * 128, 1000, page)
            self.q = (C.byref(self.g), FAR, T * Hq * 128, Hq * 128, T)
            self.T, self.rows, self.k, self.page, self.width = T, rows, k, page, -(-rows // page)
            self.rest = (None, FAR, None, None, 0, 0x100000, 1 << 50, None)      # scores, out, lse, pred, scratch as large as any, stream

        def prompt(self):
            return lib.rk_prompt_attn(*self.q, self.kv, FAR, None, self.rows, *self.rest)

        def paged(self):
            return lib.rk_paged_attn(*self.q, C.byref(self.pages), FAR, self.width, FAR, None, self.rows, *self.rest)

        def prefix(self, shared=512):
            return lib.rk_prefix_attn(*self.q, C.byref(self.pages), FAR, -(-shared // self.page), FAR, shared, FAR, self.width, FAR, None, self.rows, *self.rest)

        def sparse(self):
            return lib.rk_sparse_attn(*self.q, C.byref(self.pages), FAR, self.width, FAR, self.k, FAR, None, *self.rest)

        def select(self, n):
            return lib.rk_page_select(C.byref(self.g), FAR, n, self.T, self.page, FAR, None, self.k, 0, 1, FAR, None, 0, None)
    return Calls


# 2^24 and more rows of queries (batch * new tokens * query heads)
PREFILLS = [(64, 32, 8, 8192, 8192), (4, 32, 8, 131072, 131072), (16, 32, 8, 32768, 32768), (1, 28, 4, 600000, 600000), (300, 64, 8, 4096, 4096), (1000, 8, 8, 5000, 5000), (65535, 8, 1, 600, 600)]


@pytest.mark.parametrize("shape", PREFILLS, ids=str)
def test_whole_prompts(calls, shape):
    """What rk_prompt_attn takes over rows one behind the other is taken over pages; behind a prefix and over chosen pages likewise."""
    x = calls(*shape)
    B, Hq, H, T, _ = shape
    assert B * T * Hq >= 1 << 24
    assert x.prompt() != UNSUPPORTED and x.paged() != UNSUPPORTED and x.prefix() != UNSUPPORTED
    assert (x.sparse() == UNSUPPORTED) == (B * T * H > (2 ** 32 - 1) // 256)


@pytest.mark.parametrize("n,threads", [(1, 64), (640, 64), (641, 64), (1024, 64), (1025, 256), (4096, 256), (4097, 1024), (16384, 1024), (16385, 256)])
def test_selection(calls, n, threads):
    """As many rows of scores as the form that is launched has room for."""
    most = (2 ** 32 - 1) // threads                                              # of batch * new tokens * KV heads
    assert calls(1, 1, 1, most, 512).select(n) != UNSUPPORTED
    assert calls(1, 1, 1, most + 1, 512).select(n) == UNSUPPORTED
    assert calls(16, 32, 8, 32768, 32768).select(n) == (UNSUPPORTED if threads == 1024 else calls(1, 1, 1, 1, 16).select(n))


def test_what_no_launch_holds_is_refused(calls):
    """Workgroups of 128 query rows to a KV head (256 where two rounds of those come together), of a token and KV head over chosen pages; the join has a workgroup to a row."""
    most = (2 ** 32 - 1) // 256
    assert calls(65535, 1, 1, 256 * 256, 65536).paged() != UNSUPPORTED and calls(65535, 1, 1, 256 * 256 + 1, 65537).paged() == UNSUPPORTED
    assert calls(1, 1, 1, most, 1 << 25).sparse() != UNSUPPORTED and calls(1, 1, 1, most + 1, 1 << 25).sparse() == UNSUPPORTED
    assert calls(1, 1, 1, most, 1 << 25).prefix() != UNSUPPORTED and calls(1, 1, 1, most + 1, 1 << 25).prefix() == UNSUPPORTED
