"""mixkvq_verify_draft on the GPU against its definition in exact arithmetic (binary64 sums in order)."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def _reference(p, q, draft, n_seq, u, u_next):
    B, n1, V = p.shape
    stay, tokens = [], []
    for b in range(B):
        i = 0
        while i < n_seq[b]:
            t = draft[b, i]
            qt = (float(q[b, i, t]) if q is not None else 1.0) if 0 <= t < V else 0.0
            if not (0 <= t < V and float(u[b, i]) * qt < float(p[b, i, t])):
                break
            i += 1
        w = np.maximum(p[b, i].astype(np.float64), 0.0)
        if i < n_seq[b]:
            less = q[b, i].astype(np.float64) if q is not None else np.eye(1, V, draft[b, i])[0] if 0 <= draft[b, i] < V else np.zeros(V)
            rest = np.maximum(p[b, i].astype(np.float64) - less, 0.0)
            w = rest if rest.sum() > 0 else w
        upto = np.cumsum(w)
        over = np.nonzero(upto > float(u_next[b]) * upto[-1])[0]
        some = np.nonzero(w > 0)[0]
        t = over[0] if len(over) else some[-1] if len(some) else 0
        stay.append(i)
        tokens.append(list(draft[b, :i]) + [t] + [-1] * (n1 - 1 - i))
    return np.array(stay), np.array(tokens)


def _softmax(x):
    e = np.exp(x - x.max(-1, keepdims=True))
    return (e / e.sum(-1, keepdims=True)).astype(np.float32)


def _inputs(rng, B, n, V, onehot, sharp=3.0, near=0.5):
    logits = sharp * rng.standard_normal((B, n + 1, V))
    p, q = _softmax(logits), _softmax(logits[:, :n] + near * rng.standard_normal((B, n, V)))
    draft = np.array([[rng.choice(V, p=q[b, i] / q[b, i].astype(np.float64).sum()) for i in range(n)] for b in range(B)]).reshape(B, n)
    return p, (None if onehot else q), draft.astype(np.int32), rng.random((B, n), dtype=np.float32), rng.random(B, dtype=np.float32)


def _run(p, q, draft, u, u_next, n_seq=None, **kw):
    import paper_2512_19206_amd as M
    d = lambda a: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda()
    s = None if n_seq is None else d(np.array(n_seq, dtype=np.int32))
    stay, tokens = M.mixkvq_verify_draft(d(p), d(draft), d(u), d(u_next), p_draft=d(q), n_seq=s, **kw)
    return stay.cpu().numpy(), tokens.cpu().numpy()


@pytest.mark.parametrize("onehot", [False, True])
@pytest.mark.parametrize("B,n,V", [(1, 1, 1), (1, 4, 2), (3, 0, 100), (5, 3, 1000), (2, 64, 257), (4, 7, 2047), (4, 5, 4096), (3, 2, 4097),
                                   (130, 1, 63), (2, 4, 50257), (1, 4, 152064), (65, 4, 9999)])
def test_against_the_definition(B, n, V, onehot):
    rng = np.random.default_rng(B * 1000 + n * 10 + V)
    for near in (0.1, 1.0):
        p, q, draft, u, u_next = _inputs(rng, B, n, V, onehot, near=near)
        n_seq = [n] * B if near < 1 else [int(x) for x in rng.integers(0, n + 1, B)]
        stay, tokens = _run(p, q, draft, u, u_next, n_seq=None if near < 1 else n_seq)
        want = _reference(p, q, draft, n_seq, u, u_next)
        assert np.array_equal(stay, want[0]) and np.array_equal(tokens, want[1])


def test_borders():
    """Powers of two, so that every product and sum is exact: comparisons that are equal, the first and the last token, zeros."""
    V = 8192
    p = np.full((6, 3, V), 2.0 ** -13, dtype=np.float32)
    q = np.full((6, 2, V), 2.0 ** -13, dtype=np.float32)
    draft = np.tile(np.array([[5, 8191]], dtype=np.int32), (6, 1))
    u = np.full((6, 2), 0.5, dtype=np.float32)
    u_next = np.array([0.0, 0.5, 1.0 - 2.0 ** -13, np.nextafter(np.float32(1), np.float32(0)), 1.0, 0.25], dtype=np.float32)
    q[1, 0, 5] = 2.0 ** -12                      # u q = p: rejected
    q[2, 1, 8191] = 2.0                          # the second one rejected
    p[3, 2] = 0.0                                # nothing to draw from: token 0
    p[4, 2, 100:] = 0.0                          # u = 1: the last token with a weight
    p[5, 0, 5] = 0.0
    q[5, 0] = 1.0                                # rejected, and no remainder: drawn from p
    want = _reference(p, q, draft, [2] * 6, u, u_next)
    assert list(want[0]) == [2, 0, 1, 2, 2, 0]
    stay, tokens = _run(p, q, draft, u, u_next)
    assert np.array_equal(stay, want[0]) and np.array_equal(tokens, want[1])


def test_tokens_outside_the_vocabulary_and_lengths_outside_the_range():
    rng = np.random.default_rng(3)
    p, q, draft, u, u_next = _inputs(rng, 4, 3, 500, False, near=0.01)
    u[:] = 0.0
    draft[0, 1], draft[1, 0], draft[2, 2] = -1, 500, 2 ** 31 - 1
    for qq in (q, None):
        want = _reference(p, qq, draft, [3, 3, 3, 0], u, u_next)
        assert list(want[0]) == [1, 0, 2, 0]
        stay, tokens = _run(p, qq, draft, u, u_next, n_seq=[99, 3, 3, -5])
        assert np.array_equal(stay, want[0]) and np.array_equal(tokens, want[1])


def test_strided_probabilities_and_given_outputs():
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(4)
    p, q, draft, u, u_next = _inputs(rng, 3, 4, 3001, False)
    want = _reference(p, q, draft, [4] * 3, u, u_next)
    wide_p = torch.full((5, 3, 3008), float("nan"), device="cuda")
    wide_p[:, :, 3:3004] = torch.from_numpy(p).cuda().transpose(0, 1)
    wide_q = torch.full((3, 4, 3003), float("nan"), device="cuda")
    wide_q[..., 1:3002] = torch.from_numpy(q).cuda()
    d = lambda a: torch.from_numpy(a).cuda()
    stay, tokens = torch.full((3,), 9, dtype=torch.int32, device="cuda"), torch.full((3, 5), 9, dtype=torch.int32, device="cuda")
    got = M.mixkvq_verify_draft(wide_p[:, :, 3:3004].transpose(0, 1), d(draft), d(u), d(u_next), p_draft=wide_q[..., 1:3002],
                                n_accepted=stay, tokens=tokens)
    assert got[0] is stay and got[1] is tokens
    assert np.array_equal(stay.cpu().numpy(), want[0]) and np.array_equal(tokens.cpu().numpy(), want[1])


def test_captured_and_on_two_streams():
    import paper_2512_19206_amd as M
    rng = np.random.default_rng(6)
    d = lambda a: torch.from_numpy(a).cuda()
    sets = []
    for _ in range(2):
        p, q, draft, u, u_next = _inputs(rng, 4, 4, 40000, False)
        sets.append(((d(p), d(draft), d(u), d(u_next)), d(q), _reference(p, q, draft, [4] * 4, u, u_next)))
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[M.mixkvq_verify_draft(*a, p_draft=q, stream=s) for a, q, _ in (x,)] for _ in range(5) for x, s in zip(sets, streams)]
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        for stay, tokens in g:
            assert np.array_equal(stay.cpu().numpy(), sets[i % 2][2][0]) and np.array_equal(tokens.cpu().numpy(), sets[i % 2][2][1])
    args, q, want = sets[0]
    args = [t.clone() for t in args]
    q = q.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        stay, tokens = M.mixkvq_verify_draft(*args, p_draft=q)
    for i in (0, 1, 0):
        for dst, src in zip(list(args) + [q], list(sets[i][0]) + [sets[i][1]]):
            dst.copy_(src)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(stay.cpu().numpy(), sets[i][2][0]) and np.array_equal(tokens.cpu().numpy(), sets[i][2][1])
