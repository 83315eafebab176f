"""mixkvq_chunk_path without a launch: no handle, a new cache, and calls that have nothing to do."""
import ctypes as C

import pytest


@pytest.fixture(scope="module")
def M():
    import os
    import paper_2512_19206_amd as M
    if not os.path.exists(M.LIB_PATH):
        from paper_2512_19206_amd.build import build_library
        build_library()
    return M


def test_no_call_has_been_made(M):
    at, lib, h = 0x100000000000, M.load_library(), C.c_void_p()      # (an address that nothing may touch)
    assert lib.mixkvq_chunk_path(None) == -1
    cfg = M.make_config(B=2, Hq=4, Hkv=2, D=128, T_max=256, Gk=128, Gv=128, R=128, k4=16, k16=0)
    bufs = M.binding.Buffers(*(at + (i << 34) for i in range(5)))
    assert lib.mixkvq_cache_create(C.byref(cfg), C.byref(bufs), C.byref(h)) == 0
    st = (C.c_int64 * 3)(2048, 128, 512)
    for n_seq in ((0, 0), (0, 5)):      # nothing to do; more tokens than there are
        lib.mixkvq_chunk_attention(h, at, st, at, at, st, 4, (C.c_int32 * 2)(*n_seq), at, st, at, 0.0, 0, None, 0, None)
        assert lib.mixkvq_chunk_path(h) == 0
    lib.mixkvq_cache_destroy(h)
