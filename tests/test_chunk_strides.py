"""Strides of dimensions that have one element: nothing is reached by them, and tensors come with any."""
import ctypes as C

import numpy as np
import pytest
import torch

AT = 0x100000000000                      # (an address that nothing may touch)


@pytest.fixture(scope="module")
def M():
    import os
    import paper_2512_19206_amd as M
    if not os.path.exists(M.LIB_PATH):
        from paper_2512_19206_amd.build import build_library
        build_library()
    return M


@pytest.mark.parametrize("B,Hq,Hkv,n,q_strides,kv_strides,rc", [
    (1, 4, 2, 3, (3, 128, 512), (5, 128, 256), 0), (2, 4, 2, 1, (512, 128, 7), (256, 128, 1 << 40), 0),
    (2, 1, 1, 3, (512, 1, 128), (512, 3, 128), 0), (1, 1, 1, 1, (1, 1, 1), (9, 9, 9), 0),
    (2, 4, 2, 3, (513, 128, 512), (512, 128, 256), -1), (1, 4, 1, 3, (1, 4, 512), (1, 1, 128), -1), (1, 1, 1, 3, (1, 1, 129), (1, 1, 128), -1),
    (2, 4, 1, 3, (512, 128, 512), (512, 1, 132), -1), (1, 4, 2, 3, (3, 128, 512), (1, 129, 256), -1),
])
def test_what_the_library_accepts(M, B, Hq, Hkv, n, q_strides, kv_strides, rc):
    lib, h = M.load_library(), C.c_void_p()
    cfg = M.make_config(B=B, Hq=Hq, Hkv=Hkv, D=128, T_max=256, Gk=128, Gv=128, R=128, k4=16, k16=0)
    bufs = M.binding.Buffers(*(AT + (i << 34) for i in range(5)))
    assert lib.mixkvq_cache_create(C.byref(cfg), C.byref(bufs), C.byref(h)) == 0
    i64 = lambda x: (C.c_int64 * 3)(*x)
    # (no sequence has a token: the call ends behind its checks)
    assert lib.mixkvq_chunk_attention(h, AT, i64(q_strides), AT, AT, i64(kv_strides), n, (C.c_int32 * B)(*[0] * B), AT, i64(q_strides), AT,
                                      0.0, 0, None, 0, None) == rc
    lib.mixkvq_cache_destroy(h)


@pytest.mark.gpu
@pytest.mark.parametrize("B,Hq,Hkv,n", [(1, 4, 1, 5), (2, 2, 1, 1), (1, 1, 1, 1), (1, 2, 2, 1), (1, 1, 1, 3)])
def test_tensors_with_other_strides_there(M, B, Hq, Hkv, n):
    rng = np.random.default_rng(61)
    gc = M.Cache(M.make_config(B=B, Hq=Hq, Hkv=Hkv, D=128, T_max=256, Gk=128, Gv=128, R=128, k4=16, k16=0))
    new = lambda heads: torch.from_numpy(rng.standard_normal((B, heads, n, 128)).astype(np.float16)).cuda()
    gc.quantize_append(torch.randn(B, Hkv, 200, 128, device="cuda").half(), torch.randn(B, Hkv, 200, 128, device="cuda").half())
    q, k, v = new(Hq), new(Hkv), new(Hkv)
    want = M.mixkvq_chunk_attention(gc, q, k, v)

    def odd(t, by):      # the same elements, with strides that mean nothing where a dimension has one of them
        return torch.as_strided(t, t.shape, [s if d > 1 else by + i for i, (d, s) in enumerate(zip(t.shape, t.stride()))])

    got = M.mixkvq_chunk_attention(gc, odd(q, 3), odd(k, 11), odd(v, 7001), out=odd(torch.empty_like(q), 5))
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
