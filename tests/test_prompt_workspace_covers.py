"""rk_prompt_workspace_bytes against what the launch asks for (no GPU needed): the size for (n, L) is enough for every call of up to n tokens
and L rows, whatever form and split such a call takes."""
import ctypes as C

import pytest

LENGTHS = [1, 31, 100, 128, 129, 500, 511, 513, 1000, 2047, 2049, 4000, 8192, 32768, 131072]
TOKENS = [1, 2, 3, 4, 5, 16, 17, 31, 33, 64, 100, 127, 129, 300, 1000, 4096]
# batch, query heads, KV heads: one pair to more than twice the compute units, ragged batches and such that are too large for sharing by length
GEOMS = [(1, 1, 1), (1, 8, 1), (1, 32, 8), (2, 32, 8), (3, 28, 4), (4, 32, 8), (8, 32, 8), (16, 32, 8), (31, 8, 2), (32, 32, 8), (33, 32, 8), (64, 32, 8), (65, 32, 8),
         (64, 28, 4), (127, 4, 4), (129, 2, 2), (300, 2, 2), (513, 1, 1)]
FAR = 0x10000                                                                    # never read: without a GPU no launch begins, and a refusal comes before it


@pytest.fixture(scope="module")
def calls():
    """refused(geometry, tokens, rows, cap, bytes): does a call turn down so small a workspace?  size(geometry, tokens, rows): what is said to be enough."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("calls with made-up addresses are for machines without a GPU")
    import paper_2411_05787_amd as rk
    from paper_2411_05787_amd.binding import _Geom, _Kv, _PromptScores

    def refused(geom, n, rows, cap, nbytes):
        B, Hq, H = geom
        scores = _PromptScores(cap, None, None, None)
        kv = _Kv(FAR, FAR, H * 131072 * 128, 131072 * 128, 131072)
        g = _Geom(B, Hq, H, 128, 0.1)
        return rk.lib.rk_prompt_attn(C.byref(g), FAR, n * Hq * 128, Hq * 128, n, kv, FAR, None, rows, C.byref(scores), FAR, None, None, 0, 0x100000, nbytes, None) == -3

    def size(geom, n, rows):
        return rk.rk_prompt_workspace_bytes(rk.Geom(*geom, 128, 0.1), n, rows)
    return refused, size


@pytest.mark.parametrize("geom", GEOMS, ids=str)
def test_every_smaller_call_fits(calls, geom):
    """Each call against the sizes for its own (n, L), for the next larger ones and for the largest."""
    refused, size = calls
    asked = False
    for i, n in enumerate(TOKENS):
        for j, rows in enumerate(LENGTHS):
            if n > rows:
                continue
            over = {size(geom, TOKENS[x], LENGTHS[y]) for x in (i, min(i + 1, len(TOKENS) - 1), len(TOKENS) - 1) for y in (j, min(j + 1, len(LENGTHS) - 1), len(LENGTHS) - 1)}
            for cap in (0.0, 30.0):
                for nbytes in over:
                    assert not refused(geom, n, rows, cap, nbytes), (geom, n, rows, cap, nbytes)
                asked = asked or refused(geom, n, rows, cap, 0)
    assert asked == (geom[0] * geom[2] <= 256)                                   # (with more pairs nothing is ever split)
