"""Every form of mixkvq_chunk_attention's kernels: blocks of query rows, steps of channel places, the fp16 tier, value groups, with and
without splits, equal and ragged batches; and what their running references and records of very different scales have to carry through
several packed records of one wavefront.  Each test says which form it is about and holds the call to it."""
import numpy as np
import pytest
import torch

from chunk_strict import strict_reference
from oracle import mixkvq_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import gpu_common
    return gpu_common


def _batch(H, B, Hkv, g, K, V, lengths, **kw):
    """A cache of B sequences whose KV head j holds one of the contents K, V [C, T, D]: number (b + j) % C, cut to lengths[b % len].
    Returns it and a function (b, j) -> that pair's dequantized keys and values."""
    import paper_2512_19206_amd as M
    C, T = K.shape[:2]
    gc = M.Cache(M.make_config(B=B, Hq=Hkv * g, Hkv=Hkv, D=128, **kw))
    which = (np.arange(B)[:, None] + np.arange(Hkv)) % C
    Kd, Vd = H.dev(K), H.dev(V)
    at = torch.from_numpy(which).cuda()
    if len(lengths) == 1:
        gc.quantize_append(Kd[at][:, :, :lengths[0]].contiguous(), Vd[at][:, :, :lengths[0]].contiguous())
    else:
        for b in range(B):
            n = lengths[b % len(lengths)]
            gc.quantize_append_seq(b, Kd[at[b], :n].contiguous(), Vd[at[b], :n].contiguous())
    held = {}
    for n in set(lengths):
        oc = O.OracleCache(O.OracleConfig(B=C, Hq=g, Hkv=1, D=128, **kw))
        oc.append(K[:, None, :n], V[:, None, :n])
        assert oc.n_quant > 0
        held[n] = [oc.dequantized(i) for i in range(C)]
    return gc, lambda b, j: held[lengths[b % len(lengths)]][which[b, j]]


def _check(dequantized, g, q, k, v, out, lse, n_seq, pairs, scale, rounded_keys, tail):
    worst = 0.0
    for b, j in sorted(set(pairs)):
        n = n_seq[b]
        if n == 0:
            continue
        K0, V0 = dequantized(b, j)
        hs = slice(j * g, (j + 1) * g)
        x = [t[b, s, :n].cpu().numpy().astype(np.float64) for t, s in ((q, hs), (k, j), (v, j))]
        o, l, err, lerr = strict_reference(K0, np.clip(V0, -65504.0, 65504.0), *x, scale, 2.0 ** -11, rounded_keys, tail)
        d = np.abs(out[b, hs, :n].float().cpu().numpy() - o)
        assert np.all(d <= err), (b, j, float((d / err).max()), int((d > err).sum()), float(d.max()))
        assert np.all(np.abs(lse[b, hs, :n].cpu().numpy() - l) <= lerr), (b, j)
        worst = max(worst, float((d / err).max()))
    return worst


def _new(rng, B, heads, n, scale=1.0):
    return torch.from_numpy((rng.standard_normal((B, n, heads, 128)) * scale).astype(np.float16)).cuda().transpose(1, 2)


def _contents(rng, C, T):
    return ((rng.standard_normal((C, T, 128)) * rng.uniform(0.3, 8, 128)).astype(np.float16),
            (rng.standard_normal((C, T, 128)) * rng.uniform(0.5, 2, (C, T, 1))).astype(np.float16))


# (four steps of channel places, five, and the fp16 tier with either)
LAYOUTS = [dict(k4=16, k16=0), dict(k4=0, k16=0), dict(k4=24, k16=0), dict(k4=0, k16=12), dict(k4=24, k16=8)]


def _forty_eight(k4, k16, Gv):
    return k16 == 0 and k4 in (0, 16) and Gv == 128


@pytest.mark.parametrize("ragged", [False, True])
@pytest.mark.parametrize("n", [2, 3, 5])
@pytest.mark.parametrize("Gv", [128, 64, 32])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_row_blocks_over_every_layout(H, layout, Gv, n, ragged):
    """64 sequences, 14, 21 and 35 query rows of a KV head: one block of 16, two (the second one ragged), three or two tiles of two."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(51)
    B, Hkv, g = 64, 4, 7
    K, V = _contents(rng, 2, 470)
    gc, deq = _batch(H, B, Hkv, g, K, V, [470, 320, 90] if ragged else [470], T_max=512, R=64, Gk=64 if Gv == 128 else 32, Gv=Gv, **layout)
    q, k, v = _new(rng, B, Hkv * g, n, 2.0), _new(rng, B, Hkv, n, 2.0), _new(rng, B, Hkv, n)
    n_seq = [n - b % 2 for b in range(B)] if ragged else [n] * B
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq if ragged else None)
    assert gc.chunk_path() == {2: 16, 3: 32, 5: 48 if _forty_eight(Gv=Gv, **layout) else 32}[n]
    _check(deq, g, q, k, v, out, lse, n_seq, [(0, 0), (1, 1), (2, 2), (17, 3), (62, 1), (63, 3)], 1 / np.sqrt(128.0), False, 2.0 ** -33)


@pytest.mark.parametrize("Gv", [128, 64, 32])
@pytest.mark.parametrize("layout", LAYOUTS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_split_rows_over_every_layout(H, layout, Gv):
    """40 query rows of a KV head over 8000 tokens in several splits: two tiles of 32 rows for 8 sequences, of 48 for 24 where there are such."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(52)
    Hkv, g, n, T = 4, 8, 5, 8000
    K, V = _contents(rng, 1, T)
    for B, rows in ((8, 32), (24, 48)):
        if rows == 48 and not _forty_eight(Gv=Gv, **layout):
            continue
        gc, deq = _batch(H, B, Hkv, g, K, V, [T], T_max=8192, R=64, Gk=64 if Gv == 128 else 32, Gv=Gv, **layout)
        q, k, v = _new(rng, B, Hkv * g, n, 2.0), _new(rng, B, Hkv, n, 2.0), _new(rng, B, Hkv, n)
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
        assert gc.chunk_path() == rows and gc.lib.mixkvq_chunk_workspace(gc.handle, n, None) > 0
        _check(deq, g, q, k, v, out, lse, [n] * B, [(0, 0), (B - 1, 3)], 1 / np.sqrt(128.0), False, 2.0 ** -33)


@pytest.mark.parametrize("layout", [dict(R=16, Gk=16, Gv=128), dict(R=48, Gk=48, Gv=128), dict(R=64, Gk=16, Gv=64), dict(R=64, Gk=64, Gv=16)],
                         ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
def test_layouts_that_only_the_kernel_for_many_rows_takes(H, layout):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(53)
    B, Hkv, g, n = 2, 2, 4, 2
    K, V = _contents(rng, 2, 300)
    gc, deq = _batch(H, B, Hkv, g, K, V, [300], T_max=480 if layout["R"] == 48 else 512, k4=8, k16=0, **layout)
    assert gc.chunk_path() == 0
    q, k, v = _new(rng, B, Hkv * g, n, 2.0), _new(rng, B, Hkv, n, 2.0), _new(rng, B, Hkv, n)
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
    assert gc.chunk_path() == 256
    _check(deq, g, q, k, v, out, lse, [n] * B, [(0, 0), (0, 1), (1, 0), (1, 1)], 1 / np.sqrt(128.0), True, 2.0 ** -30)


# Few rows: 14, 21 and 35 of a KV head in batches that leave every wavefront several slices; many: 560.
FORMS = [(64, 4, 7, 2, 16), (64, 4, 7, 3, 32), (64, 4, 7, 5, 48), (1, 1, 7, 80, 256)]


@pytest.mark.parametrize("B,Hkv,g,n,rows", FORMS, ids=lambda x: str(x))
@pytest.mark.parametrize("R,Gk,Gv,k4,k16", [(128, 128, 128, 16, 0), (32, 32, 128, 0, 4), (128, 32, 32, 8, 4), (32, 32, 64, 16, 0)])
@pytest.mark.parametrize("jump", [20.0, 25.0, 60.0])
def test_scores_that_jump_inside_packed_records(H, B, Hkv, g, n, rows, R, Gk, Gv, k4, k16, jump):
    """Scores (in powers of two) of 0, then of 12.9 on 24 tokens, then one of `jump` and one of twice that, over and over through 1900
    packed tokens: every wavefront meets them in its own run, and what 24 weights carry must not be lost where the sums change their
    reference."""
    import paper_2512_19206_amd as M
    if rows == 48 and not _forty_eight(k4, k16, Gv):
        rows = 32
    rng = np.random.default_rng(54)
    T = 1900
    K, V = np.zeros((1, T, 128), np.float16), rng.standard_normal((1, T, 128)).astype(np.float16)
    for t in range(0, T - 200, 190):
        K[0, t + 40:t + 64, 0], V[0, t + 40:t + 64] = 12.9, 8.0
        K[0, t + 100, 0], K[0, t + 165, 0] = jump, 2 * jump
    gc, deq = _batch(H, B, Hkv, g, K, V, [T], T_max=1920, R=R, Gk=Gk, Gv=Gv, k4=k4, k16=k16)
    q = torch.zeros(B, Hkv * g, n, 128, dtype=torch.float16, device="cuda")
    q[..., 0] = float(np.log(2.0))
    v = _new(rng, B, Hkv, n)
    k = torch.zeros_like(v)
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v, scale=1.0)
    assert gc.chunk_path() == rows
    _check(deq, g, q, k, v, out, lse, [n] * B, [(0, 0), (B - 1, Hkv - 1)], 1.0, rows == 256, 2.0 ** -30)


@pytest.mark.parametrize("B,Hkv,g,n,rows", FORMS, ids=lambda x: str(x))
@pytest.mark.parametrize("R,Gk,Gv", [(128, 128, 128), (32, 32, 128), (32, 32, 32)])
@pytest.mark.parametrize("lead", [False, True])
def test_records_of_very_different_scales(H, B, Hkv, g, n, rows, R, Gk, Gv, lead):
    """Values (and keys) whose scales change by 2^6 to 2^12 from one record to the next, up and down; with lead, a token of the first
    record has the largest score by far, so that everything else counts little."""
    import paper_2512_19206_amd as M
    if rows == 48 and Gv != 128:
        rows = 32
    rng = np.random.default_rng(55)
    T, B_ = 1900, B
    size = np.array([1.0, 64.0, 2.0 ** -6, 2048.0, 1.0, 2.0 ** -6, 4096.0, 0.25])[np.arange(T) // R % 8][None, :, None]
    V = (rng.standard_normal((1, T, 128)) * size).astype(np.float16)
    K = (rng.standard_normal((1, T, 128)) * np.minimum(size, 8.0) * 0.3).astype(np.float16)
    K[0, 5, :] = 0.0
    if lead:
        K[..., 0], V[0, 5] = 0.0, 0.0
        K[0, 5, 0] = 16.0
    gc, deq = _batch(H, B_, Hkv, g, K, V, [T], T_max=1920, R=R, Gk=Gk, Gv=Gv, k4=16, k16=0)
    q, k, v = _new(rng, B, Hkv * g, n, 0.5), _new(rng, B, Hkv, n, 0.5), _new(rng, B, Hkv, n)
    if lead:
        q[..., 0] = 8.0      # the leading score: 16 * 8 / 11.3 = 11.3, 2^16
        k[..., 0] = 0.0
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
    assert gc.chunk_path() == rows
    _check(deq, g, q, k, v, out, lse, [n] * B, [(0, 0), (B - 1, Hkv - 1)], 1 / np.sqrt(128.0), rows == 256, 2.0 ** -30)
