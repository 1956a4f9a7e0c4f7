"""rk_rope_append and rk_rope_append_q8 in place: only where q lies as q_out does (no GPU needed)."""
import ctypes as C

import pytest


@pytest.mark.parametrize("batch,n,sb,st", [(2, 3, 3 * 6144, 6144), (2, 3, 3 * 4096 + 8, 4096), (1, 3, 0, 6144), (2, 1, 6144, 0), (1, 2, 0, 0)])
def test_other_strides_are_refused(batch, n, sb, st):
    """Rows of 32 query heads inside those of a projection of 48, or repeated: their tokens would be written over one another."""
    import paper_2411_05787_amd as rk
    from paper_2411_05787_amd.binding import _Geom, _Kv, _Kv8, _NewRows, _Rope
    g, f = _Geom(batch, 32, 8, 128, 0.1), 0x10000
    rows, rope = _NewRows(f, f, f, sb, st, 0, 0, 0, 0, n), _Rope(f, 64, 128, 0)
    kv, kv8 = _Kv(f, f, 8 * 64 * 128, 64 * 128, 64), _Kv8(f, f, f, f, f, f, 8 * 64 * 128, 64 * 128, 64, 32, 0)
    assert rk.lib.rk_rope_append(C.byref(g), C.byref(rows), C.byref(rope), None, kv, f, None, f, None, 0, None) == -1
    assert rk.lib.rk_rope_append_q8(C.byref(g), C.byref(rows), C.byref(rope), None, C.byref(kv8), f, None, f, None, 0, None) == -1
