"""What mixkvq_chunk_attention and mixkvq_verify_draft refuse, and calls that have nothing to do: all of it is decided on the host, so no
pointer is ever read here."""
import ctypes as C

import pytest

EINVAL, ESCRATCH = -1, -7
AT = 0x100000000000                      # (an address that nothing may touch)
KW = dict(B=3, Hq=14, Hkv=2, D=128, T_max=4096, Gk=128, Gv=128, R=128, k4=16, k16=0)


@pytest.fixture(scope="module")
def M():
    import os
    import paper_2512_19206_amd as M
    if not os.path.exists(M.LIB_PATH):
        from paper_2512_19206_amd.build import build_library
        build_library()
    return M


@pytest.fixture()
def cache(M):
    lib, h = M.load_library(), C.c_void_p()
    cfg = M.make_config(**KW)
    bufs = M.binding.Buffers(*(AT + (i << 34) for i in range(5)))
    assert lib.mixkvq_cache_create(C.byref(cfg), C.byref(bufs), C.byref(h)) == 0
    for b, (nq, nr) in enumerate(((2048, 100), (0, 0), (128, 1))):
        assert lib.mixkvq_cache_set_state_seq(h, b, nq, nr, 0) == 0
    yield h
    lib.mixkvq_cache_destroy(h)


def _chunk(M, h, **change):
    n = change.get("n_new", 4)
    st = lambda H, m: (C.c_int64 * 3)(max(m, 1) * H * 128, 128, H * 128)
    a = dict(c=h, q=AT, q_strides=st(14, n), k=AT, v=AT, kv_strides=st(2, n), n_new=n, n_seq=None, out=AT, out_strides=st(14, n), lse=AT,
             scale=0.0, acc=0, workspace=None, bytes=0, stream=None)
    a.update(change)
    return M.load_library().mixkvq_chunk_attention(*a.values())


def _i64(*x):
    return (C.c_int64 * len(x))(*x)


def _i32(*x):
    return (C.c_int32 * len(x))(*x)


@pytest.mark.parametrize("change", [
    dict(c=None), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(q_strides=None), dict(kv_strides=None), dict(out_strides=None),
    dict(q=AT + 8), dict(k=AT + 2), dict(v=AT + 4), dict(out=AT + 8), dict(workspace=AT + 8, bytes=1 << 30),
    dict(q_strides=_i64(7168, 128, 1788)), dict(kv_strides=_i64(1024, 4, 256)), dict(out_strides=_i64(7170, 128, 1792)),
    dict(n_new=-1), dict(n_new=(1 << 20) + 1), dict(n_seq=_i32(1, 5, 2)), dict(n_seq=_i32(1, -1, 2)),
    dict(scale=float("inf")), dict(kv_strides=_i64(1024, 128, 1 << 33)),
])
def test_chunk_attention_refuses(M, cache, change):
    assert _chunk(M, cache, **dict(dict(workspace=AT, bytes=1 << 40), **change)) == EINVAL


def test_chunk_workspace(M, cache):
    lib = M.load_library()
    assert lib.mixkvq_chunk_workspace(None, 4, None) == EINVAL
    assert lib.mixkvq_chunk_workspace(cache, -1, None) == EINVAL
    assert lib.mixkvq_chunk_workspace(cache, (1 << 20) + 1, None) == EINVAL
    assert lib.mixkvq_chunk_workspace(cache, 4, _i32(0, 5, 0)) == EINVAL
    assert lib.mixkvq_chunk_workspace(cache, 0, None) == 0
    assert lib.mixkvq_chunk_workspace(cache, 4, _i32(0, 4, 0)) == 0      # (an empty cache: nothing to split)
    need = lib.mixkvq_chunk_workspace(cache, 4, None)
    assert need > 0 and need % 4 == 0
    for given in ((None, 0), (None, need), (AT, need - 1), (AT, 0)):
        assert _chunk(M, cache, workspace=given[0], bytes=given[1]) == ESCRATCH


def test_chunk_attention_without_new_tokens(M, cache):
    assert _chunk(M, cache, n_new=0) == 0
    assert _chunk(M, cache, n_seq=_i32(0, 0, 0)) == 0
    assert _chunk(M, cache, n_seq=_i32(0, 0, 0), acc=1) == 0


def _verify(M, **change):
    a = dict(B=2, n=4, V=50000, p=AT, ps=_i64(250000, 50000), q=AT, qs=_i64(200000, 50000), draft=AT, n_seq=None, u=AT, u_next=AT,
             accepted=AT, tokens=AT, workspace=AT, bytes=1 << 30, stream=None)
    a.update(change)
    return M.load_library().mixkvq_verify_draft(*a.values())


@pytest.mark.parametrize("change", [
    dict(B=0), dict(B=(1 << 20) + 1), dict(V=0), dict(V=-5), dict(n=-1), dict(n=65), dict(p=None), dict(ps=None), dict(qs=None), dict(draft=None),
    dict(u=None), dict(u_next=None), dict(accepted=None), dict(tokens=None), dict(workspace=None), dict(workspace=AT + 8),
    dict(V=(1 << 30) + 1), dict(p=AT + 2), dict(q=AT + 1), dict(draft=AT + 2), dict(n_seq=AT + 1), dict(u=AT + 2), dict(u_next=AT + 3),
    dict(accepted=AT + 2), dict(tokens=AT + 1),
])
def test_verify_draft_refuses(M, change):
    assert _verify(M, **change) == EINVAL


def test_verify_workspace(M):
    lib = M.load_library()
    for bad in ((0, 10), ((1 << 20) + 1, 10), (4, 0), (1, (1 << 30) + 1)):
        assert lib.mixkvq_verify_workspace(*bad) == EINVAL
    for B, V in ((1, 1), (2, 50000), (128, 50000), (64, 152064), (1, 1 << 30)):
        need = lib.mixkvq_verify_workspace(B, V)
        assert need >= 16 * B
        assert _verify(M, B=B, V=V, bytes=need - 1) == ESCRATCH
