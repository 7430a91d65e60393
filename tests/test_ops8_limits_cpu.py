"""Sizes past what the 8-bit operators' launches hold: refused before a launch."""
import ctypes as C

D = C.c_void_p(0x10000)      # never read: every call here ends before a launch


def test_append_refuses_more_pages_than_a_grid_holds():
    from paper_2312_04429_amd import _native as N
    for T, W in (((1 << 31) - 1, (1 << 31) - 1), ((1 << 30) - 126, 1 << 24)):
        assert N.lib.nv_op_kv8_append(D, 16, 0, D, 16, 0, N.NV_F16, 1, T, 1, 16, D, D, D, D, 4, D, W, D,
                                      None, None) == N.NV_ERR_UNSUPPORTED
