"""mixkvq_chunk_attention, mixkvq_verify_draft and the appends between them, as a serving loop runs them; and the sizes at which
addresses, row tiles and parts of a vocabulary change their form."""
import numpy as np
import pytest
import torch

from oracle import mixkvq_oracle as O
from test_gpu_chunk_attention import _kv, _new
from test_gpu_verify_draft import _inputs, _reference

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def H():
    assert torch.cuda.is_available(), "these tests need the GPU"
    import chunk_common
    import gpu_common
    gpu_common.chunk = chunk_common
    return gpu_common


@pytest.mark.parametrize("paged", [False, True])
@pytest.mark.parametrize("flush_mode", [0, 1])
def test_speculative_steps(H, paged, flush_mode):
    """Ragged sequences, a draft of 0 .. 5 tokens each: the target pass, the verdict, and the accepted tokens appended one sequence at
    a time; windows fill and are packed on the way, and every pass agrees with the formula over what was appended."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(21 + paged)
    B, Hkv, g, n, V, NB = 4, 2, 5, 5, 777, 12
    kw = dict(Hq=Hkv * g, Hkv=Hkv, D=128, T_max=NB * 32, Gk=32, Gv=32, R=32, k4=8, k16=4, sink=32, flush_mode=flush_mode)
    gc = M.Cache(M.make_config(B=B, **kw))
    if paged:
        gc.set_block_table(torch.from_numpy(rng.permutation(B * NB).astype(np.int32)).view(B, -1).cuda())
    ocs = [O.OracleCache(O.OracleConfig(B=1, **kw)) for _ in range(B)]
    for b, T in enumerate([0, 60, 126, 200]):
        if T:
            K, W = _kv(rng, 1, Hkv, T)
            gc.quantize_append_seq(b, H.dev(K)[0], H.dev(W)[0])
            ocs[b].append(K, W)
    lengths, want_lengths = [0, 60, 126, 200], [0, 60, 126, 200]
    for turn in range(14):
        drafts = [int(x) for x in rng.integers(0, n + 1, B)]
        p, pq, draft, u, u_next = _inputs(rng, B, n, V, turn % 3 == 2, near=0.2)
        q, k, v = _new(rng, B, Hkv * g, n + 1, 2.0), _new(rng, B, Hkv, n + 1, 2.0), _new(rng, B, Hkv, n + 1)
        n_seq = [m + 1 for m in drafts]
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v, n_seq=n_seq)
        H.chunk.check_chunk(lambda b: (ocs[b], 0), g, Hkv, q, k, v, n_seq, out, lse, name=f"turn {turn}")
        dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x)).cuda()
        stay, tokens = M.mixkvq_verify_draft(dev(p), dev(draft), dev(u), dev(u_next), p_draft=dev(pq), n_seq=dev(np.array(drafts, np.int32)))
        want = _reference(p, pq, draft, drafts, u, u_next)
        assert np.array_equal(stay.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])
        for b, m in enumerate(stay.tolist()):      # the last token that was there and the drafts that stay
            gc.quantize_append_seq(b, k[b, :, :m + 1], v[b, :, :m + 1])
            ocs[b].append(k[b:b + 1, :, :m + 1].cpu().numpy(), v[b:b + 1, :, :m + 1].cpu().numpy())
            lengths[b] += m + 1
            want_lengths[b] += want[0][b] + 1
    assert lengths == want_lengths and max(lengths) > 210


def test_a_prompt_in_pieces(H):
    """Attention of each piece over what was packed of the ones before it, then the piece enters the cache."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(22)
    B, Hkv, g = 2, 2, 7
    kw = dict(B=B, Hq=Hkv * g, Hkv=Hkv, D=128, T_max=1024, Gk=128, Gv=128, R=128, k4=16, k16=0)
    oc, gc = H.make_pair(**kw)
    for m in (100, 1, 27, 128, 129, 300):
        q, k, v = _new(rng, B, Hkv * g, m, 2.0), _new(rng, B, Hkv, m, 2.0), _new(rng, B, Hkv, m)
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v, accumulate_q=True)
        H.chunk.check_chunk(lambda b: (oc, b * Hkv), g, Hkv, q, k, v, [m] * B, out, lse, name=f"piece {m}")
        gc.quantize_append(k, v)
        # (queries are counted on both sides, so that the channels chosen for the next blocks agree)
        oc.accumulate_queries(q.cpu().numpy())
        oc.append(k.cpu().numpy(), v.cpu().numpy())
    H.check_state(oc, gc)


@pytest.mark.parametrize("n", [3, 9, 20, 37, 70, 74])
def test_row_tiles_of_both_kernels(H, n):
    """21 to 518 rows of a KV head: one tile, several ones of 48 or 32 rows, tiles of 256 rows, the last one ragged."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(23 + n)
    for k16, Gv, Gk in ((0, 128, 128), (8, 32, 32)):
        kw = dict(B=1, Hq=7, Hkv=1, D=128, T_max=2048, Gk=Gk, Gv=Gv, R=128, k4=16, k16=k16)
        oc, gc = H.make_pair(**kw)
        K, V = _kv(rng, 1, 1, 2000)
        gc.quantize_append(H.dev(K), H.dev(V))
        oc.append(K, V)
        q, k, v = _new(rng, 1, 7, n, 2.0), _new(rng, 1, 1, n, 2.0), _new(rng, 1, 1, n)
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
        H.chunk.check_chunk(lambda b: (oc, 0), 7, 1, q, k, v, [n], out, lse)


@pytest.mark.parametrize("T", [0, 200])
@pytest.mark.parametrize("n", [5, 300])
@pytest.mark.parametrize("jump", [20.0, 25.0, 60.0])
def test_a_largest_score_far_ahead_of_the_one_before(H, T, n, jump):
    """Scores (in powers of two) of 0, then of 12.9 on 24 tokens, then one of `jump`: what 24 weights of 2^-12.1 carry must not be lost
    where the sums change their reference."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(26)
    kw = dict(B=1, Hq=4, Hkv=1, D=128, T_max=256, Gk=128, Gv=128, R=256, k4=16, k16=0)
    oc, gc = H.make_pair(**kw)
    K, V = np.zeros((1, 1, T + n, 128), np.float16), rng.standard_normal((1, 1, T + n, 128)).astype(np.float16)
    K[0, 0, 40:64, 0], V[0, 0, 40:64] = 12.9, 8.0
    K[0, 0, 70:71, 0] = jump
    K[0, 0, -3:-2, 0] = 2 * jump
    if T:
        gc.quantize_append(H.dev(K[:, :, :T]), H.dev(V[:, :, :T]))
        oc.append(K[:, :, :T], V[:, :, :T])
    q = torch.zeros(1, 4, n, 128, dtype=torch.float16, device="cuda")
    q[..., 0] = float(np.log(2.0))
    k, v = H.dev(K[:, :, T:]), H.dev(V[:, :, T:])
    out, lse = M.mixkvq_chunk_attention(gc, q, k, v, scale=1.0)
    H.chunk.check_chunk(lambda b: (oc, 0), 4, 1, q, k, v, [n], out, lse, scale=1.0)


@pytest.mark.parametrize("paged", [False, True])
def test_records_beyond_four_gigabytes(H, paged):
    """The last KV heads' records start past 2^32 bytes (and, by a table, at the end of the pool)."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(24)
    Hkv, g, T, NB = 8, 2, 700, 65536
    kw = dict(B=1, Hq=Hkv * g, Hkv=Hkv, D=128, Gk=128, Gv=128, R=128, k4=16, k16=0)
    gc = M.Cache(M.make_config(T_max=NB * 128, **kw))
    assert 7 * NB * gc.layout.rec_bytes > 1 << 32
    if paged:
        gc.set_block_table(torch.arange(NB - 1, -1, -1, dtype=torch.int32).view(1, -1).cuda())
    oc = O.OracleCache(O.OracleConfig(T_max=1024, **kw))
    K, V = _kv(rng, 1, Hkv, T)
    gc.quantize_append(H.dev(K), H.dev(V))
    oc.append(K, V)
    for n in (4, 150):
        q, k, v = _new(rng, 1, Hkv * g, n, 2.0), _new(rng, 1, Hkv, n, 2.0), _new(rng, 1, Hkv, n)
        out, lse = M.mixkvq_chunk_attention(gc, q, k, v)
        H.chunk.check_chunk(lambda b: (oc, 0), g, Hkv, q, k, v, [n], out, lse)


@pytest.mark.parametrize("B,n,V", [(130, 2, 20000), (128, 1, 65536), (2, 1, 65537), (1, 1, 1300001), (3, 0, 16385), (2, 64, 17000)])
@pytest.mark.parametrize("onehot", [False, True])
def test_verdicts_on_vocabularies_of_every_form(B, n, V, onehot):
    """One launch for many rows, two for few; more than 4096 tokens in a part."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(B + n + V)
    rows = min(B, 3)      # (sequences repeat: the reference is slow)
    p, q, draft, u, u_next = _inputs(rng, rows, n, V, onehot, near=0.5)
    want = _reference(p, q, draft, [n] * rows, u, u_next)
    at = np.arange(B) % rows
    dev = lambda x: None if x is None else torch.from_numpy(np.ascontiguousarray(x[at])).cuda()
    stay, tokens = M.mixkvq_verify_draft(dev(p), dev(draft), dev(u), dev(u_next), p_draft=dev(q))
    assert np.array_equal(stay.cpu().numpy(), want[0][at]) and np.array_equal(tokens.cpu().numpy(), want[1][at])


def test_the_last_tokens_are_drawn_at_the_ends_of_parts():
    """u = 0 takes the first token with a weight, u just below 1 the last one, wherever it stands."""
    import paper_2512_19206_amd as M
    for V in (300, 16384, 50001, 1300001):
        spots = sorted({0, 1, V // 4 - 1, V // 4, V // 2 + 3, V - 2, V - 1})
        p = torch.zeros(len(spots), 1, V, device="cuda")
        for i, s in enumerate(spots):
            p[i, 0, s] = 0.25
        dev = dict(device="cuda")
        for u in (0.0, 0.5, 1.0 - 2.0 ** -24, 1.0):
            stay, tokens = M.mixkvq_verify_draft(p, torch.zeros(len(spots), 0, dtype=torch.int32, **dev), torch.zeros(len(spots), 0, **dev),
                                                 torch.full((len(spots),), u, **dev))
            assert stay.tolist() == [0] * len(spots) and tokens[:, 0].tolist() == spots
        p.zero_()
        assert M.mixkvq_verify_draft(p, torch.zeros(len(spots), 0, dtype=torch.int32, **dev), torch.zeros(len(spots), 0, **dev),
                                     torch.full((len(spots),), 0.5, **dev))[1].flatten().tolist() == [0] * len(spots)


def test_calls_on_host_tensors_are_refused(H):
    """Before anything is launched."""
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(25)
    gc = M.Cache(M.make_config(B=1, Hq=2, Hkv=1, D=128, T_max=64, Gk=32, Gv=32, R=32, k4=8, k16=0))
    q, k, v = _new(rng, 1, 2, 3), _new(rng, 1, 1, 3), _new(rng, 1, 1, 3)
    for i in range(3):
        a = [q, k, v]
        a[i] = a[i].cpu()
        with pytest.raises(AssertionError):
            M.mixkvq_chunk_attention(gc, *a)
    for kw in (dict(out=torch.empty_like(q, device="cpu")), dict(lse=torch.empty(1, 2, 3)), dict(workspace=torch.empty(1 << 20, dtype=torch.uint8))):
        with pytest.raises(AssertionError):
            M.mixkvq_chunk_attention(gc, q, k, v, **kw)
    p, pq, draft, u, u_next = (torch.from_numpy(x).cuda() for x in _inputs(rng, 2, 3, 50, False))
    good = dict(p_target=p, draft=draft, u_accept=u, u_next=u_next, p_draft=pq, n_seq=torch.tensor([3, 2], dtype=torch.int32, device="cuda"))
    M.mixkvq_verify_draft(**good)
    for name in good:
        with pytest.raises(AssertionError):
            M.mixkvq_verify_draft(**dict(good, **{name: good[name].cpu()}))
    for kw in (dict(n_accepted=torch.empty(2, dtype=torch.int32)), dict(tokens=torch.empty(2, 4, dtype=torch.int32)),
               dict(workspace=torch.empty(1 << 16, dtype=torch.uint8))):
        with pytest.raises(AssertionError):
            M.mixkvq_verify_draft(**good, **kw)
