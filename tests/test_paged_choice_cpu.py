"""The knob that chooses the kernel of attention over a paged cache takes its three values and no other."""
import ctypes



def test_paged_dense_knob(libdodo):
    from paper_2310_02409_b200 import api
    lib, c = api.load(), ctypes.c_void_p()
    lib.dodo_create(ctypes.byref(c), 0)
    try:
        assert [lib.dodo_set_tuning(c, api.TUNE_PAGED_DENSE, v) for v in (1, 2, 0)] == [api.OK] * 3
        assert [lib.dodo_set_tuning(c, api.TUNE_PAGED_DENSE, v) for v in (-1, 3)] == [api.ERR_INVALID_ARG] * 2
        assert lib.dodo_set_tuning(c, 2, 0) == api.ERR_INVALID_ARG and lib.dodo_set_tuning(c, 6, 0) == api.ERR_INVALID_ARG
    finally:
        lib.dodo_destroy(c)
