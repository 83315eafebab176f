"""mixkvq_chunk_attention on the GPU against the formula in 64 bits over the oracle's cache."""
import numpy as np
import pytest
import torch

from oracle import mixkvq_oracle as O

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import chunk_common
    import gpu_common
    gpu_common.chunk = chunk_common
    return gpu_common


def _new(rng, B, heads, n, scale=1.0, dtype=torch.float16, layout="bnhd"):
    """[B, heads, n, D] on the GPU, stored as [B, n, heads, D] (layout "bnhd"), or with its heads outermost and gaps ("gaps")."""
    x = torch.from_numpy((rng.standard_normal((B, n, heads, 128)) * scale).astype(np.float32)).to(dtype).cuda()
    if layout == "bnhd":
        return x.transpose(1, 2)
    wide = torch.full((heads, B, n + 2, 136), float("nan"), dtype=dtype, device="cuda")
    wide[:, :, :n, :128] = x.permute(2, 0, 1, 3)
    return wide[:, :, :n, :128].transpose(0, 1)


def _kv(rng, B, Hkv, n):
    K = (rng.standard_normal((B, Hkv, n, 128)) * rng.uniform(0.3, 8, 128)).astype(np.float16)
    return K, rng.standard_normal((B, Hkv, n, 128)).astype(np.float16)


BASE = dict(B=2, Hkv=2, g=4, R=128, Gk=128, Gv=128, k4=16, k16=0, T=300, n=5)
CASES = [
    dict(n=1), dict(n=8, T=0), dict(n=33, T=7), dict(n=16, T=128), dict(n=17, T=129), dict(n=32, T=257), dict(n=64, T=1),
    dict(n=65, T=640), dict(n=130, T=385, B=1), dict(n=300, T=0, B=1, Hkv=1, g=3),
    dict(g=7, n=9, T=700), dict(g=1, n=1, T=130), dict(g=8, n=16, T=300), dict(g=5, n=51, T=300, B=1), dict(g=8, n=8), dict(g=1, n=65),
    dict(R=32, Gk=32, Gv=32, k4=8, T=333), dict(R=32, Gk=16, Gv=16, k4=8, k16=4, T=201), dict(R=64, Gk=64, Gv=64, T=513),
    dict(R=64, Gk=32, Gv=32, k4=0, k16=12, T=400), dict(R=128, Gk=32, Gv=64, k4=16, k16=8, T=513),
    dict(R=256, Gk=128, Gv=128, T=1100), dict(R=16, Gk=16, Gv=128, T=100), dict(R=48, Gk=48, Gv=32, T=300), dict(R=80, Gk=16, Gv=64, T=300),
    dict(R=96, Gk=32, Gv=128, T=400), dict(R=96, Gk=96, Gv=128, T=400), dict(R=112, Gk=16, Gv=16, T=400, n=20),
    dict(k4=0, k16=0, T=513), dict(k4=8, k16=48, Gk=64, T=300), dict(k4=120, k16=4, Gk=32, Gv=16, T=300),
    dict(sink=64, R=64, Gk=32, Gv=64, T=300), dict(sink=128, T=40, n=12), dict(sink=32, T=700, flush_mode=1),
    dict(policy=1, tau16=20.0, tau4=4.0, k16=8, Gk=32, Gv=32, T=700), dict(policy=1, tau16=1.0, tau4=0.0, k16=12, k4=112, T=400),
    dict(policy=1, tau16=float("inf"), tau4=float("inf"), k16=4, k4=8, R=32, Gk=32, Gv=32, T=300),
    dict(dtype="bf16", n=11), dict(dtype="bf16", n=130, T=300, B=1), dict(layout="gaps", n=7), dict(layout="gaps", n=70, dtype="bf16"),
    dict(scale=0.02, n=9), dict(T=4000, n=3, B=1, Hkv=1, g=5),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()))
@pytest.mark.parametrize("paged", [False, True])
def test_against_the_formula(H, case, paged):
    import paper_2512_19206_amd as M
    c = dict(BASE, **case)
    if paged and c["T"] < c["R"]:
        pytest.skip("no record")
    rng = np.random.default_rng(sum(map(ord, repr(sorted(case.items())))))
    B, Hkv, g, n, T, scale = c["B"], c["Hkv"], c["g"], c.pop("n"), c.pop("T"), c.pop("scale", 0.0)
    dt = torch.bfloat16 if c.pop("dtype", "f16") == "bf16" else torch.float16
    layout = c.pop("layout", "bnhd")
    c["Hq"] = c.pop("g") * Hkv
    kw = dict(c, D=128, T_max=-(-max(T, 1) // c["R"]) * c["R"])
    oc = O.OracleCache(O.OracleConfig(**kw))
    gc = M.Cache(M.make_config(in_dtype=int(dt == torch.bfloat16), **kw))
    if paged:
        slots = B * (kw["T_max"] // gc.rec_tokens)
        gc.set_block_table(torch.from_numpy(rng.permutation(slots).astype(np.int32)).view(B, -1).cuda())
    if T:
        K, V = _kv(rng, B, Hkv, T)
        Kd, Vd = torch.from_numpy(K).cuda().to(dt), torch.from_numpy(V).cuda().to(dt)
        gc.quantize_append(Kd, Vd)
        oc.append(H.chunk.kept(Kd).astype(np.float16), H.chunk.kept(Vd).astype(np.float16))
    q = _new(rng, B, Hkv * g, n, rng.uniform(0.2, 4, 128), dt, layout)
    k, v = _new(rng, B, Hkv, n, 2.0, dt, layout), _new(rng, B, Hkv, n, 1.0, dt, layout)
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v, scale=scale)
    assert out.shape == q.shape and out.dtype == dt
    H.chunk.check_chunk(lambda b: (oc, b * Hkv), g, Hkv, q, k, v, [n] * B, out, lse, scale=scale, name=repr(case))
    if not paged and dt == torch.float16:
        H.check_state(oc, gc)      # the cache is as it was


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_sequences_and_chunks_of_different_lengths(H, paged, dtype):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(77 + paged)
    B, Hkv, g, R, n = 6, 2, 7, 64, 40
    kw = dict(Hq=Hkv * g, Hkv=Hkv, D=128, T_max=16 * R, Gk=32, Gv=64, R=R, k4=8, k16=4)
    gc = M.Cache(M.make_config(B=B, in_dtype=int(dtype == torch.bfloat16), **kw))
    if paged:
        gc.set_block_table(torch.from_numpy(rng.permutation(B * 16).astype(np.int32)).view(B, -1).cuda())
    ocs = [O.OracleCache(O.OracleConfig(B=1, **kw)) for _ in range(B)]
    for b, T in enumerate([1000, 0, 64, 65, 17, 500]):
        if T:
            K, V = _kv(rng, 1, Hkv, T)
            Kd, Vd = torch.from_numpy(K).cuda().to(dtype), torch.from_numpy(V).cuda().to(dtype)
            gc.quantize_append_seq(b, Kd[0], Vd[0])
            ocs[b].append(H.chunk.kept(Kd).astype(np.float16), H.chunk.kept(Vd).astype(np.float16))
    for n_seq in ([40, 40, 0, 1, 39, 7], [0, 3, 0, 0, 40, 0], [0] * B, [1] * B, [40] * B):
        q = _new(rng, B, Hkv * g, n, 2.0, dtype)
        k, v = _new(rng, B, Hkv, n, 2.0, dtype), _new(rng, B, Hkv, n, 1.0, dtype)
        for b, m in enumerate(n_seq):      # what stands behind a sequence's tokens is never read ...
            for t in (q, k, v):
                t[b, :, m:] = float("nan")
        out = torch.full_like(q, 7.0)
        lse = torch.full((B, Hkv * g, n), 7.0, device="cuda")
        M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq, out=out, lse=lse)
        H.chunk.check_chunk(lambda b: (ocs[b], 0), g, Hkv, q, k, v, n_seq, out, lse, name=str(n_seq))
        for b, m in enumerate(n_seq):      # ... and never written
            assert bool((out[b, :, m:] == 7.0).all()) and bool((lse[b, :, m:] == 7.0).all())


def test_more_sequences_than_one_launch_takes(H):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(5)
    B, Hkv, g, n = 131, 1, 3, 2
    kw = dict(B=B, Hq=g, Hkv=Hkv, D=128, T_max=64, Gk=32, Gv=32, R=32, k4=8, k16=0)
    oc, gc = O.OracleCache(O.OracleConfig(**kw)), M.Cache(M.make_config(**kw))
    K, V = _kv(rng, B, Hkv, 60)
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    q, k, v = _new(rng, B, g, n, 2.0), _new(rng, B, Hkv, n, 2.0), _new(rng, B, Hkv, n)
    n_seq = [b % 3 for b in range(B)]
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq)
    H.chunk.check_chunk(lambda b: (oc, b), g, Hkv, q, k, v, n_seq, out, lse)


def test_one_new_token_agrees_with_the_decode_step(H):
    """The same numbers by the other path: append, then attend."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(8)
    kw = dict(B=3, Hq=14, Hkv=2, D=128, T_max=1024, Gk=128, Gv=128, R=128, k4=16, k16=0)
    oc, gc = H.make_pair(**kw)
    K, V = _kv(rng, 3, 2, 900)
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    oc_before = [oc.dequantized(p) for p in range(6)]
    q, k, v = _new(rng, 3, 14, 1, 2.0), _new(rng, 3, 2, 1, 2.0), _new(rng, 3, 2, 1)
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
    ref, ref_lse = M.mixkvq_decode_step(gc, k.contiguous(), v.contiguous(), q[:, :, 0].contiguous())
    a, r = (t.float().cpu().numpy().astype(np.float64) for t in (out[:, :, 0], ref))
    al, rl = (t.cpu().numpy().astype(np.float64) for t in (lse[:, :, 0], ref_lse))
    # Scores reach 40 here, so half a step of binary16 in what they are made of moves a weight by a few percent: both are held to
    # the bound that their roundings give.  The decode kernel rounds q s instead of the key c s + z, half a step of |q| c s, and
    # c s is at most the range of the key channel.
    qh, kh, vh = (H.chunk.kept(t) for t in (q, k, v))
    for b in range(3):
        for j in range(2):
            K0, V0 = oc_before[b * 2 + j]
            hs = slice(7 * j, 7 * j + 7)
            size = np.broadcast_to(np.ptp(np.concatenate([K0, kh[b, j]]), axis=0), (K0.shape[0] + 1, 128))
            rounds = np.abs(np.concatenate([V0, vh[b, j]]))
            rounds[:-1] += V0 - V0.min(axis=1, keepdims=True)
            o, l, e1, l1 = H.chunk.chunk_reference(K0, V0, qh[b, hs], kh[b, j], vh[b, j], 1 / np.sqrt(128.0), 2.0 ** -11, rounds=rounds)
            _, _, e2, l2 = H.chunk.chunk_reference(K0, V0, qh[b, hs], kh[b, j], vh[b, j], 1 / np.sqrt(128.0), 2.0 ** -11, key_size=size, rounds=rounds)
            assert np.all(np.abs(a[b, hs] - o[:, 0]) <= e1[:, 0]) and np.all(np.abs(a[b, hs] - r[b, hs]) <= e1[:, 0] + e2[:, 0])
            assert np.all(np.abs(al[b, hs] - l[:, 0]) <= l1[:, 0]) and np.all(np.abs(al[b, hs] - rl[b, hs]) <= l1[:, 0] + l2[:, 0])


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_accumulates_the_queries_on_request(H, dtype):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(9)
    B, Hkv, g, n = 3, 2, 5, 30
    kw = dict(B=B, Hq=g * Hkv, Hkv=Hkv, D=128, T_max=64, Gk=32, Gv=32, R=32, k4=8, k16=0)
    gc = M.Cache(M.make_config(in_dtype=int(dtype == torch.bfloat16), **kw))
    q, k, v = _new(rng, B, Hkv * g, n, 3.0, dtype), _new(rng, B, Hkv, n, 1.0, dtype), _new(rng, B, Hkv, n, 1.0, dtype)
    n_seq = [30, 0, 11]
    for _ in range(2):
        M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq, accumulate_q=True)
    M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq)
    acc, cnt = (t.cpu().numpy() for t in gc.query_accumulator())
    qh = H.chunk.kept(q)
    for b in range(B):
        for j in range(Hkv):
            want = np.abs(qh[b, j * g:(j + 1) * g, :n_seq[b]]).sum((0, 1)) * 2.0 ** 24 * 2
            assert np.array_equal(acc[b * Hkv + j], want.astype(np.int64))
            assert cnt[b * Hkv + j] == 2 * g * n_seq[b]


def test_large_values_stay_finite(H):
    """Groups whose dequantized values reach the end of binary16, constant groups, zeros; bfloat16 tensors beyond its range."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(10)
    kw = dict(B=1, Hq=2, Hkv=1, D=128, T_max=128, Gk=32, Gv=32, R=32, k4=8, k16=4)
    K, V = _kv(rng, 1, 1, 100)
    V[..., :40] *= 0
    V[0, 0, ::2, 64:96] = 65504.0
    V[0, 0, 1::2, 64:96] = np.where(rng.random((50, 32)) < 0.5, 65504.0, -65504.0)
    K[..., 5] = 3.0
    K[..., 6] = 0.0
    oc, gc = H.make_pair(**kw)
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    q, k, v = _new(rng, 1, 2, 6, 0.3), _new(rng, 1, 1, 6), _new(rng, 1, 1, 6)
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
    K0, V0 = oc.dequantized(0)
    o, l, err, lerr = H.chunk.chunk_reference(K0, np.clip(V0, -65504.0, 65504.0), *(H.chunk.kept(t)[0] for t in (q,)),
                                              H.chunk.kept(k)[0, 0], H.chunk.kept(v)[0, 0], 1 / np.sqrt(128.0), 2.0 ** -11)
    got = out.float().cpu().numpy()[0]
    assert np.all(np.isfinite(got)) and np.all(np.abs(got - o) <= err)

    gb = M.Cache(M.make_config(in_dtype=1, **kw))
    q, k, v = (_new(rng, 1, h, 6, s, torch.bfloat16) for h, s in ((2, 0.3), (1, 1.0), (1, 1.0)))
    v[0, 0, 2, 7], v[0, 0, 3, 7], k[0, 0, 1, 3] = 3e38, -1e30, 1e5
    out, lse = M.mixkvq_chunk_attention(gb, q, k, v)
    empty = O.OracleCache(O.OracleConfig(**kw))
    H.chunk.check_chunk(lambda b: (empty, 0), 2, 1, q, k, v, [6], out, lse)


def test_equal_scores_and_far_apart_scores(H):
    """Zero queries (every token weighs the same), and scores that grow along the tokens by far more than the kernel's headroom."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(11)
    kw = dict(B=1, Hq=4, Hkv=1, D=128, T_max=512, Gk=128, Gv=128, R=128, k4=16, k16=0)
    oc, gc = H.make_pair(**kw)
    K, V = _kv(rng, 1, 1, 500)
    K[0, 0, :, 0] = np.linspace(-100, 100, 500)
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    q, k, v = _new(rng, 1, 4, 50), _new(rng, 1, 1, 50), _new(rng, 1, 1, 50)
    q[0, 0] = 0.0
    q[0, 1, :, 0] = 60.0
    q[0, 2, :, 0] = -60.0
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
    H.chunk.check_chunk(lambda b: (oc, 0), 4, 1, q, k, v, [50], out, lse)


def _filled(M, H, rng, B=2, T=2000, g=7, Hkv=2, dtype=torch.float16):
    kw = dict(B=B, Hq=Hkv * g, Hkv=Hkv, D=128, T_max=2048, Gk=128, Gv=128, R=128, k4=16, k16=0)
    gc = M.Cache(M.make_config(in_dtype=int(dtype == torch.bfloat16), **kw))
    K, V = _kv(rng, B, Hkv, T)
    gc.quantize_append(H.dev(K).to(dtype), H.dev(V).to(dtype))
    return gc


def test_captured_graphs_replayed_between_eager_calls(H):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(12)
    gc = _filled(M, H, rng)
    sets = [[_new(rng, 2, h, 9) for h in (14, 2, 2)] for _ in range(3)]
    want = [M.mixkvq_chunk_attention(gc, *s)[0].clone() for s in sets]
    q, k, v = (t.clone() for t in sets[0])
    q2, k2, v2 = (t.clone() for t in sets[1])
    graphs = []
    for a in ((q, k, v), (q2, k2, v2)):      # two graphs, each with the workspace of its own call
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out, _ = M.mixkvq_chunk_attention(gc, *a)
        graphs.append((g, out))
    for i in (0, 1, 2, 0, 2):
        for dst, src in ((q, sets[i][0]), (k, sets[i][1]), (v, sets[i][2])):
            dst.copy_(src)
        for dst, src in zip((q2, k2, v2), sets[(i + 1) % 3]):
            dst.copy_(src)
        for g, _ in graphs:
            g.replay()
        eager = M.mixkvq_chunk_attention(gc, *sets[i])[0]
        torch.cuda.synchronize()
        assert torch.equal(graphs[0][1], want[i]) and torch.equal(graphs[1][1], want[(i + 1) % 3]) and torch.equal(eager, want[i])


def test_two_streams_at_once_and_the_same_bits_every_time(H):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(13)
    gc = _filled(M, H, rng)
    sets = [[_new(rng, 2, h, n) for h in (14, 2, 2)] for n in (5, 40)]
    want = [M.mixkvq_chunk_attention(gc, *s)[0].clone() for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for i, s in enumerate(streams):
            got[i].append(M.mixkvq_chunk_attention(gc, *sets[i], stream=s)[0])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i]) for o in got[i])


def test_gaps_of_a_wide_output_are_left_alone(H):
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(14)
    gc = _filled(M, H, rng)
    for n in (3, 50):
        q, k, v = (_new(rng, 2, h, n) for h in (14, 2, 2))
        wide = torch.full((2, n + 3, 14, 144), 9.0, dtype=torch.float16, device="cuda")
        out = wide[:, :n, :, 8:136].transpose(1, 2)
        M.mixkvq_chunk_attention(gc, q, k, v, out=out)
        want = M.mixkvq_chunk_attention(gc, q, k, v)[0]
        assert torch.equal(out, want)
        assert bool((wide[:, n:] == 9.0).all()) and bool((wide[..., :8] == 9.0).all()) and bool((wide[..., 136:] == 9.0).all())


def test_a_long_prompt_in_pieces_and_at_once(H):
    """Pieces attend over packed blocks, so only a prompt that stays in the window gives the same numbers; a long piece over an
    empty cache is checked against float64 on the GPU."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(15)
    B, Hkv, g, n = 1, 2, 4, 1500
    kw = dict(B=B, Hq=Hkv * g, Hkv=Hkv, D=128, T_max=2048, Gk=128, Gv=128, R=256, k4=16, k16=0)
    gc = M.Cache(M.make_config(**kw))
    q, k, v = _new(rng, B, Hkv * g, n), _new(rng, B, Hkv, n), _new(rng, B, Hkv, n)
    whole = M.mixkvq_chunk_attention(gc, q, k, v)[0]
    for h in range(Hkv * g):
        s = (q[0, h].double() @ k[0, h // g].double().T) / np.sqrt(128.0)
        s = torch.softmax(s.masked_fill(torch.ones(n, n, device="cuda").triu(1).bool(), -float("inf")), -1)
        ref = s @ v[0, h // g].double()
        # unit normal inputs: |s| <= 15, so a score is off by at most 15 * 2^-11 * 3 and the output by twice that of |v| <= 6 (weights)
        assert float((whole[0, h].double() - ref).abs().max()) <= 2 * 6 * (15 * 3 + 4) * 2.0 ** -11
        assert float((whole[0, h].double() - ref).norm() / ref.norm()) <= 4 * 2.0 ** -11 * 3
    at = 0
    for m in (100, 1, 27, 128):
        piece = M.mixkvq_chunk_attention(gc, q[:, :, at:at + m], k[:, :, at:at + m], v[:, :, at:at + m])[0]
        assert bool(((piece.float() - whole[:, :, at:at + m].float()).abs() <= 2e-3 + 1e-2 * whole[:, :, at:at + m].float().abs()).all())
        gc.quantize_append(k[:, :, at:at + m], v[:, :, at:at + m])
        at += m
