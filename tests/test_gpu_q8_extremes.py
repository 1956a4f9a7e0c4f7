"""The cache of 8 bits where a block's largest value is at the ends of bf16's range: bit for bit oracle/new_tokens.py's, and back out of it."""
import sys

import numpy as np
import pytest
import torch

import gen
from oracle import new_tokens as o

pytestmark = pytest.mark.gpu

# bits of the largest magnitude of each block: the largest finite values, the formats' own mantissas around the step of the scale, the smallest
# normal values, subnormal ones
TOPS = [0x7f7f, 0x7f7e, 0x7f61, 0x7f60, 0x7f5f, 0x7f00, 0x7eff, 0x0101, 0x0100, 0x00ff, 0x0080, 0x007f, 0x0060, 0x0002, 0x0001]


@pytest.fixture(scope="module")
def rk():
    import paper_2411_05787_amd as lib
    return lib


@pytest.mark.parametrize("block", [16, 128])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_blocks_at_the_ends_of_the_range(rk, fmt, block):
    print("ends of the range", fmt, block, file=sys.stderr, flush=True)
    n, r = len(TOPS) * block, np.random.default_rng(4)
    b = np.zeros((n, 128), np.int64)
    for i, top in enumerate(TOPS):                                               # magnitudes near the largest, far below it and anywhere between
        m = np.where(r.random((block, 128)) < 0.5, r.integers(max(top - 0x500, 0), top + 1, (block, 128)), r.integers(0, top + 1, (block, 128)))
        m[r.integers(block), r.integers(128)] = top
        b[i * block:(i + 1) * block] = m | (r.integers(0, 2, (block, 128)) << 15)
    bits = b.astype(np.uint16)
    rows = torch.from_numpy(bits.view(np.int16).copy()).view(torch.bfloat16).view(1, n, 1, 128).cuda()
    dtype = torch.float8_e4m3fn if fmt == "e4m3" else torch.int8
    geom = rk.Geom(1, 1, 1, 128, 0.1)
    cache = rk.Kv8.empty(geom, n, block, dtype)
    lens = torch.tensor([n], dtype=torch.int32, device="cuda")
    rk.rk_rope_append_q8(geom, None, rows, rows, None, cache, lens, None)
    small = [torch.zeros(1, 1, n, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    rk.rk_gather_small_kv_q8(geom, cache, torch.arange(n, dtype=torch.int32, device="cuda").view(1, 1, n), n, *small, lens)
    torch.cuda.synchronize()
    x = o.bf16_bits_to_f64(bits)
    for t, s, back in ((cache.k, cache.k_scale, small[0]), (cache.v, cache.v_scale, small[1])):
        got, back = t.view(torch.uint8).cpu().view(dtype).double().numpy()[0, 0], gen.bf16_bits(back)[0, 0]
        for i in range(len(TOPS)):
            at = slice(i * block, (i + 1) * block)
            want, scale = o.quantise_block(x[at], fmt)
            assert float(s[0, 0, i]) == scale, (hex(TOPS[i]), float(s[0, 0, i]), scale)
            assert (got[at] == want).all(), hex(TOPS[i])
            # back out of it: the product rounded to bf16 (a subnormal one may lose bits); 2^128, where a largest value was rounded up, is an infinity
            y = want * scale
            big = np.abs(y) >= 2.0 ** 128
            exact = o.bf16_bits_to_f64(o.f64_to_bf16_bits(np.where(big, 0.0, y)))
            np.testing.assert_array_equal(o.bf16_bits_to_f64(back[at]), np.where(big, np.copysign(np.inf, y), exact), err_msg=hex(TOPS[i]))
