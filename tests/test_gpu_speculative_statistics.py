"""A speculative loop that keeps the statistics of the queries: |q| of the tokens that stay enters the accumulator before they are appended,
that of rejected drafts never does, and the channels of every packed block follow from it."""
import numpy as np
import pytest
import torch

from oracle import mixkvq_oracle as O
from test_gpu_chunk_attention import _new
from test_gpu_ragged import _check_seq
from test_gpu_verify_draft import _inputs

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import chunk_common
    import gpu_common
    gpu_common.chunk = chunk_common
    return gpu_common


@pytest.mark.parametrize("policy", [0, 1])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_only_what_stays_is_counted(H, policy, dtype):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(71)
    B, Hkv, g, n, V = 3, 2, 5, 4, 500
    kw = dict(Hq=Hkv * g, Hkv=Hkv, D=128, T_max=256, Gk=32, Gv=128, R=32, k4=8, k16=4)
    if policy:
        kw.update(policy=1, tau16=4.0, tau4=2.0)
    gc = M.Cache(M.make_config(B=B, in_dtype=int(dtype == torch.bfloat16), **kw))
    ocs = [O.OracleCache(O.OracleConfig(B=1, **kw)) for _ in range(B)]
    half = lambda t: H.chunk.kept(t).astype(np.float16)
    loud = rng.permutation(np.concatenate([np.full(12, 6.0), np.full(116, 0.5)]))      # channels that the queries are large in
    stayed, rejected = 0, 0
    for turn in range(30):
        p, pq, draft, u, u_next = _inputs(rng, B, n, V, False, near=0.3)
        q = _new(rng, B, Hkv * g, n + 1, loud if turn % 2 else 1.0, dtype)
        k, v = _new(rng, B, Hkv, n + 1, 1.5, dtype), _new(rng, B, Hkv, n + 1, 1.0, dtype)
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
        H.chunk.check_chunk(lambda b: (ocs[b], 0), g, Hkv, q, k, v, [n + 1] * B, out, lse, name=f"turn {turn}")
        dev = lambda x: torch.from_numpy(np.ascontiguousarray(x)).cuda()
        stay, _ = M.mixkvq_verify_draft(dev(p), dev(draft), dev(u), dev(u_next), p_draft=dev(pq))
        for b, m in enumerate(stay.tolist()):
            gc.select_channels_seq(b, q[b, :, :m + 1], k[b, :, :m + 1])
            gc.quantize_append_seq(b, k[b, :, :m + 1], v[b, :, :m + 1])
            ocs[b].accumulate_queries(half(q[b:b + 1, :, :m + 1]))
            ocs[b].append(half(k[b:b + 1, :, :m + 1]), half(v[b:b + 1, :, :m + 1]))
            stayed, rejected = stayed + m + 1, rejected + n - m
    assert stayed > 100 and rejected > 100
    for b in range(B):
        assert ocs[b].n_quant > 0 and ocs[b].qacc.any()
        _check_seq(H, gc, b, ocs[b], Hkv)
