"""Sequences without new tokens before, between and behind others whose tokens are split over workgroups: they own no split, their outputs
stay as they were, and the others' do not depend on them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n", [4, 100])      # few and many query rows of a KV head
def test_idle_sequences_in_a_split_batch(n):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(81)
    B, Hkv, g, T = 9, 2, 6, 3000
    gc = M.Cache(M.make_config(B=B, Hq=Hkv * g, Hkv=Hkv, D=128, T_max=3200, Gk=128, Gv=128, R=128, k4=16, k16=0))
    half = lambda *shape: torch.from_numpy(rng.standard_normal(shape).astype(np.float16)).cuda()
    for b in range(B):
        m = T - 317 * b
        gc.quantize_append_seq(b, half(Hkv, m, 128), half(Hkv, m, 128))
    q, k, v = half(B, Hkv * g, n, 128), half(B, Hkv, n, 128), half(B, Hkv, n, 128)
    idle = {0, 3, 4, 7, 8}
    n_seq = [0 if b in idle else n for b in range(B)]
    assert gc.lib.mixkvq_chunk_workspace(gc.handle, n, (M.binding.C.c_int32 * B)(*n_seq)) > 0
    out, lse = torch.full_like(q, 7.0), torch.full((B, Hkv * g, n), 7.0, device="cuda")
    M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq, out=out, lse=lse)
    alone, alone_lse = M.mixkvq_chunk_attention(gc, q, k, v)
    for b in range(B):
        if b in idle:
            assert bool((out[b] == 7.0).all()) and bool((lse[b] == 7.0).all())
        else:      # (the batch may be cut otherwise: weights in binary16 relative to other references, outputs of at most 1)
            assert float((out[b].float() - alone[b].float()).abs().max()) <= 2 * 2.0 ** -11 * 4
            assert float((lse[b] - alone_lse[b]).abs().max()) <= 2 * 2.0 ** -11
