"""mixkvq_chunk_attention over value groups in which one element lies far from the others (Eq. 3: x~ = c s + z with |z| >> |x~| for the
ordinary elements): what the kernels round may only be relative to the values, not to c s or z, as it is for one token at a time."""
import numpy as np
import pytest
import torch

from chunk_strict import strict_reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import gpu_common
    return gpu_common


@pytest.mark.parametrize("focus", [0.0, 0.35])
@pytest.mark.parametrize("X", [8.0, 300.0, 512.0, 2000.0, 65504.0])
# (few query rows of a KV head, 14, and many, 560)
@pytest.mark.parametrize("n,G,k4,k16", [(2, 128, 16, 0), (2, 128, 0, 12), (2, 64, 16, 0), (2, 32, 16, 0), (80, 128, 16, 0), (80, 32, 16, 0)])
def test_one_far_element_per_value_group(H, n, G, focus, X, k4, k16):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(31)
    T, g = 700, 7
    oc, gc = H.make_pair(B=1, Hq=g, Hkv=1, D=128, T_max=1024, Gk=G, Gv=G, R=128, k4=k4, k16=k16)
    K = rng.standard_normal((1, 1, T, 128)).astype(np.float16)
    V = rng.standard_normal((1, 1, T, 128)).astype(np.float16)
    for t in range(0, T, 5):                       # every fifth token: one element of each value group is -X or +X
        for g0 in range(0, 128, G):
            V[0, 0, t, g0 + (t % G)] = -X if (t // 5) % 2 == 0 else X
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    assert oc.n_quant == 640
    q = rng.standard_normal((1, g, n, 128)).astype(np.float16)
    if focus:                                      # rows that lean on one such token each, with weights well below 1
        for h in range(g):
            for i in range(n):
                q[0, h, i] = (K[0, 0, 5 * ((h + 7 * i) % 128)].astype(np.float32) * focus + q[0, h, i]).astype(np.float16)
    k, v = (rng.standard_normal((1, 1, n, 128)).astype(np.float16) for _ in range(2))
    out, lse = M.mixkvq_chunk_attention(gc, H.dev(q), H.dev(k), H.dev(v))
    K0, V0 = oc.dequantized(0)
    o, l, err, lerr = strict_reference(K0, np.clip(V0, -65504.0, 65504.0), *(x.astype(np.float64) for x in (q[0], k[0, 0], v[0, 0])),
                                       1 / np.sqrt(128.0), 2.0 ** -11, rounded_keys=n > 2, tail=2.0 ** -24)
    d = np.abs(out[0].float().cpu().numpy() - o)
    assert np.all(d <= err), (float((d / err).max()), int((d > err).sum()), float(d.max()))
    assert np.all(np.abs(lse[0].cpu().numpy() - l) <= lerr)
    if n == 2:      # and the bar that a decode step meets on the same cache (few rows take the queries times scales to 22 bits)
        assert np.all(d <= H.value_atol(X) + H.RTOL * np.abs(o)), float((d - H.RTOL * np.abs(o)).max())
