"""Serving several new tokens of a sequence at once over the quantized cache, as cases that can be timed and compared.

Two operators:

  chunk     attention of n new tokens per sequence over what the cache holds of it (packed records, then fp16 rows) and
            over the chunk itself, causally: a piece of a long prompt, or the drafted tokens of a speculative step.
  verify    the drafted tokens against the target's probabilities with given random numbers: how many stay, and the
            token that follows them.

The cache's contents are made here as the bytes of its documented record layout (packed codes, scales, zero-points),
so that both forms read the same records.  The plain forms are elementary torch operations in 32 bits, the verification's
in 64 (its sums run over the whole vocabulary and are compared with a random number).
"""
import math

import numpy as np
import torch

own = False

D = 128


def _cfg(hq, hkv, R=128, G=128, k4=16, k16=0, thresholds=False, dtype="f16"):
    return dict(hq=hq, hkv=hkv, R=R, G=G, k4=k4, k16=k16, thresholds=thresholds, dtype=dtype)


def listed():
    return [
        # The first speculative step after a short prompt: everything still sits in the fp16 window.
        dict(name="chunk_b1_window", kind="chunk", B=1, T=90, T_min=90, n=5, n_min=5, paged=False, **_cfg(28, 4)),
        # The smallest quantized cache, one head, an odd number of drafted tokens.
        dict(name="chunk_b1_1k", kind="chunk", B=1, T=1027, T_min=1027, n=7, n_min=7, paged=False,
             **_cfg(1, 1, R=32, G=32, k4=8)),
        # A speculative step (four drafted tokens and the last accepted one) on the benchmark's headline batch.
        dict(name="chunk_b8_32k", kind="chunk", B=8, T=32805, T_min=32805, n=5, n_min=5, paged=False, **_cfg(28, 4)),
        # The same for a large batch with the fp16 tier.
        dict(name="chunk_b64_32k", kind="chunk", B=64, T=32790, T_min=32790, n=4, n_min=4, paged=False,
             **_cfg(40, 8, k4=0, k16=12)),
        # Long reasoning with longer drafts, paged records.
        dict(name="chunk_b4_128k_paged", kind="chunk", B=4, T=131091, T_min=131091, n=9, n_min=9, paged=True,
             **_cfg(40, 8)),
        # Continuous batching: contexts and drafts of very different lengths, thresholds, bfloat16 tensors, paged records.
        dict(name="chunk_b24_ragged_paged", kind="chunk", B=24, T=12003, T_min=60, n=16, n_min=1, paged=True,
             **_cfg(28, 4, G=32, k4=16, k16=8, thresholds=True, dtype="bf16")),
        # A later piece of a long prompt behind its packed prefix.
        dict(name="chunk_b1_1000_of_32k", kind="chunk", B=1, T=31000, T_min=31000, n=1000, n_min=1000, paged=False,
             **_cfg(28, 4, dtype="bf16")),
        # Prompt pieces of two requests with the short residual window.
        dict(name="chunk_b2_2048_of_10k", kind="chunk", B=2, T=8190, T_min=8190, n=2048, n_min=2048, paged=False,
             **_cfg(40, 8, R=32, G=32)),
        # A whole prompt into an empty cache.
        dict(name="chunk_b1_8192_first", kind="chunk", B=1, T=0, T_min=0, n=8192, n_min=8192, paged=False, **_cfg(28, 4)),
        # One sequence's drafts, a small vocabulary.
        dict(name="verify_b1_32k", kind="verify", B=1, n=4, n_min=4, V=32000, onehot=False),
        # Drafts without probabilities (looked up in the prompt), as many as each sequence found; an odd vocabulary.
        dict(name="verify_b16_50k_onehot", kind="verify", B=16, n=8, n_min=0, V=50257, onehot=True),
        # A large batch over a large vocabulary.
        dict(name="verify_b64_152k", kind="verify", B=64, n=4, n_min=4, V=152064, onehot=False),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges."""
    if rng.random() < 0.25:
        B, n = _log_int(rng, 1, 64), rng.randint(1, 10)
        return dict(kind="verify", B=B, n=n, n_min=n if rng.random() < 0.5 else rng.randint(0, n), V=_log_int(rng, 1000, 152064),
                    onehot=rng.random() < 0.4)
    hq, hkv = rng.choice([(1, 1), (14, 2), (28, 4), (40, 8), (40, 8), (28, 4), (8, 8)])
    R, G = rng.choice([(128, 128), (128, 128), (128, 128), (128, 32), (128, 64), (64, 64), (32, 32), (256, 128)])
    k4, k16, thr = rng.choice([(16, 0, False), (16, 0, False), (0, 12, False), (8, 0, False), (16, 8, True)])
    base = _cfg(hq, hkv, R=R, G=G, k4=k4, k16=k16, thresholds=thr, dtype=rng.choice(["f16", "bf16"]))
    if rng.random() < 0.6:        # a speculative step
        B, n = _log_int(rng, 1, 64), rng.randint(1, 24)
        T = _log_int(rng, 40, min(131072, 16 * 8 * 32768 // (B * hkv)))
        ragged = B > 1 and rng.random() < 0.5
        return dict(kind="chunk", B=B, T=T, T_min=_log_int(rng, 1, T) if ragged else T, n=n, n_min=rng.randint(0, n) if ragged else n,
                    paged=rng.random() < 0.5, **base)
    B, n = rng.choice([1, 1, 2, 3]), _log_int(rng, 30, 3000)
    T = 0 if rng.random() < 0.25 else _log_int(rng, 100, 16000)
    n = min(n, max(30, int(2e9 // (B * hq * (T + n)))))
    return dict(kind="chunk", B=B, T=T, T_min=T, n=n, n_min=n, paged=rng.random() < 0.3, **base)


# ---------------------------------------------------------------------------- the record layout

def _al16(n):
    return -(-n // 16) * 16


def _layout(case):
    """Planes of one record: name -> (byte offset, element type, shape)."""
    Rr = min(case["R"], 128)
    Gk, Gv, k4, k16 = min(case["G"], Rr), case["G"], case["k4"], case["k16"]
    NL = D if case["thresholds"] else D - k4 - k16
    NLp, NG = _al16(NL), Rr // Gk
    planes, off = {}, 0
    for name, dt, shape in (("idx", torch.uint8, (k16 + k4,)), ("kmax", torch.float16, (NG + 1,)),
                            ("lo_s", torch.float16, (NG, NLp)), ("lo_z", torch.float16, (NG, NLp)),
                            ("k4_s", torch.float16, (NG, k4)), ("k4_z", torch.float16, (NG, k4)),
                            ("lo", torch.int32, (Rr, NLp // 16)), ("k4", torch.int32, (Rr, k4 // 8)),
                            ("k16", torch.float16, (Rr, k16)), ("v", torch.int32, (Rr // 16, D)),
                            ("v_s", torch.float16, (Rr, D // Gv)), ("v_z", torch.float16, (Rr, D // Gv))):
        planes[name] = (off, dt, shape)
        off += _al16(math.prod(shape) * dt.itemsize)
    return dict(planes=planes, rec_bytes=off, Rr=Rr, Gk=Gk, Gv=Gv, NLp=NLp, NL=NL, NG=NG, k4=k4, k16=k16,
                interleave=Gk == 32 and Rr % 64 == 0)


def _plane(records, lay, name):
    """records [..., rec_bytes] -> that plane of every record, [..., *shape]."""
    off, dt, shape = lay["planes"][name]
    n = math.prod(shape)
    return records[..., off:off + n * dt.itemsize].contiguous().view(dt).view(records.shape[:-1] + shape)


# ---------------------------------------------------------------------------- inputs

def _spread(lo, hi, B):
    """B whole numbers from lo to hi, in no order."""
    return [int(round(lo + (hi - lo) * ((0.618034 * (b + 1)) % 1.0))) for b in range(B)]


def _lengths(case):
    """Context length and number of new tokens of every sequence (contexts spread over their logarithm)."""
    lo = max(1, case["T_min"])
    T = [case["T"]] * case["B"] if case["T_min"] == case["T"] else \
        [int(round(lo * (case["T"] / lo) ** ((0.381966 * (b + 1)) % 1.0))) for b in range(case["B"])]
    n = _spread(case["n_min"], case["n"], case["B"])
    if case["n"] not in n:
        n[0] = case["n"]
    return T, n


def _counts(T, R):
    """(packed tokens, tokens in the fp16 window) of a sequence of T tokens."""
    packed = (max(T, 1) - 1) // R * R
    return packed, T - packed


def _heavy_tail(shape, gen):
    """|t| with 3 degrees of freedom, unit mean: magnitudes of tokens."""
    z = torch.randn((4,) + shape, generator=gen, device="cuda")
    return z[0].abs() / (z[1:].square().sum(0) / 3.0).sqrt() / 1.1027


def _outliers(shape, gen):
    """[..., D] channel scales: 1, except 4 channels at 10 to 20."""
    c = torch.ones(shape + (D,), device="cuda")
    at = torch.rand(shape + (D,), generator=gen, device="cuda").topk(4, dim=-1).indices
    return c.scatter_(-1, at, 10.0 + 10.0 * torch.rand(shape + (4,), generator=gen, device="cuda"))


def _words(shape, gen):
    return torch.randint(-(1 << 31), 1 << 31, shape, generator=gen, device="cuda", dtype=torch.int32)


def _two_bit(shape, gen):
    """Words of 16 two-bit codes spread as those of normal values: 1/16, 7/16, 7/16, 1/16."""
    hi, a = _words(shape, gen), _words(shape, gen) | _words(shape, gen) | _words(shape, gen)
    return (hi & -0x55555556) | (((hi >> 1) ^ a) & 0x55555555)


def _four_bit(shape, gen):
    """Words of 8 four-bit codes, the mean of two uniform ones."""
    a, b = _words(shape, gen), _words(shape, gen)
    return (a & b) + (((a ^ b) >> 1) & 0x77777777)


def _put(records, lay, name, value):
    off, dt, shape = lay["planes"][name]
    n = math.prod(shape)
    if n:
        records[..., off:off + n * dt.itemsize] = value.to(dt).expand(records.shape[:-1] + shape).contiguous().view(
            records.shape[:-1] + (n,)).view(torch.uint8)


def _records(case, lay, kc, nb, gen):
    """nb records of every KV head of one sequence, uint8 [nb, Hkv, rec_bytes]; kc [Hkv, D]: scale of the key channels."""
    H, k4, k16, NG, Gk, Rr = kc.shape[0], lay["k4"], lay["k16"], lay["NG"], lay["Gk"], lay["Rr"]
    rec = torch.zeros((nb, H, lay["rec_bytes"]), dtype=torch.uint8, device="cuda")
    # channels by a noisy score: one choice for the sequence, or one for every record under the thresholds, of which the
    # tiers then hold different numbers
    per = nb if case["thresholds"] else 1
    order = (kc * torch.exp(0.5 * torch.randn((per, H, D), generator=gen, device="cuda"))).argsort(dim=-1, descending=True)
    if case["thresholds"]:
        n16 = torch.randint(0, k16 + 1, (per, H, 1), generator=gen, device="cuda")
        n4 = torch.randint(0, k4 + 1, (per, H, 1), generator=gen, device="cuda")
    else:
        n16, n4 = torch.full((1, H, 1), k16, device="cuda"), torch.full((1, H, 1), k4, device="cuda")
    at = torch.arange(D, device="cuda").expand(per, H, D)
    tier = torch.empty_like(order).scatter_(-1, order, (at >= n16).long() + (at >= n16 + n4).long())
    lists = [(torch.where(tier == i, at, at + 1024).sort(dim=-1).values)[..., :w] for i, w in ((0, k16), (1, k4), (2, lay["NLp"]))]
    used16, used4, used = (x < D for x in lists)
    chans = [x.clamp(max=D - 1) for x in lists]
    _put(rec, lay, "idx", torch.cat([torch.where(x < D, x, 255) for x in lists[:2]], dim=-1))
    # scales follow the channel and the largest token of the group; zero-points put the codes around zero
    c16, c4, clo = (torch.gather(kc.expand(per, H, D), -1, x) for x in chans)
    mag = (_heavy_tail((nb, H, NG, 8), gen).amax(dim=-1) * 0.8 + 1.0)[..., None]
    lo_s = (clo[:, :, None] * mag * (1.4 + 0.4 * torch.rand((nb, H, NG, lay["NLp"]), generator=gen, device="cuda")) * used[:, :, None]).half()
    lo_z = lo_s.float() * (-1.5 + 0.2 * torch.randn(lo_s.shape, generator=gen, device="cuda"))
    _put(rec, lay, "lo_s", lo_s)
    _put(rec, lay, "lo_z", lo_z)
    words = _two_bit((nb, H, Rr, lay["NLp"] // 16), gen)
    bits = torch.tensor([3 << (16 * (i & 1) + 2 * (i >> 1)) for i in range(16)], device="cuda")
    keep = (used.view(per, H, 1, -1, 16) * bits).sum(-1)
    _put(rec, lay, "lo", words & torch.where(keep >= 1 << 31, keep - (1 << 32), keep).int())
    biggest = lo_s.float().amax(dim=-1)
    if k4:
        s = (c4[:, :, None] * mag * (0.28 + 0.08 * torch.rand((nb, H, NG, k4), generator=gen, device="cuda")) * used4[:, :, None]).half()
        _put(rec, lay, "k4_s", s)
        _put(rec, lay, "k4_z", s.float() * (-7.5 + torch.randn(s.shape, generator=gen, device="cuda")))
        bits = torch.tensor([15 << (16 * (i & 1) + 4 * (i >> 1)) for i in range(8)], device="cuda")
        keep = (used4.view(per, H, 1, -1, 8) * bits).sum(-1)
        _put(rec, lay, "k4", _four_bit((nb, H, Rr, k4 // 8), gen) & torch.where(keep >= 1 << 31, keep - (1 << 32), keep).int())
        biggest = torch.maximum(biggest, s.float().amax(dim=-1))
    if k16:
        x = torch.randn((nb, H, Rr, k16), generator=gen, device="cuda") * _heavy_tail((nb, H, Rr, 1), gen)
        _put(rec, lay, "k16", (x * c16[:, :, None]).clamp(-32768.0, 32768.0) * used16[:, :, None])
    _put(rec, lay, "v", _two_bit((nb, H, Rr // 16, D), gen))
    v_s = (_heavy_tail((nb, H, Rr, 1), gen) * (1.4 + 0.4 * torch.rand((nb, H, Rr, D // lay["Gv"]), generator=gen, device="cuda"))).half()
    _put(rec, lay, "v_s", v_s)
    _put(rec, lay, "v_z", v_s.float() * (-1.5 + 0.2 * torch.randn(v_s.shape, generator=gen, device="cuda")))
    _put(rec, lay, "kmax", torch.cat([biggest, v_s.float().amax(dim=(-2, -1))[..., None]], dim=-1))
    return rec


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def _prepare_chunk(case, gen):
    B, H, Hq, R, n = case["B"], case["hkv"], case["hq"], case["R"], case["n"]
    lay, dt = _layout(case), _dtype(case)
    T, n_seq = _lengths(case)
    counts = [_counts(t, R) for t in T]
    NB = max(1, -(-max(c[0] for c in counts) // lay["Rr"]))
    NB = -(-(NB * lay["Rr"]) // R) * R // lay["Rr"]                  # capacity in records, whole blocks
    table = None
    if case["paged"]:
        table = torch.randperm(B * NB, generator=gen, device="cuda").int().view(B, NB).contiguous()
        store = torch.zeros((B * NB, H, lay["rec_bytes"]), dtype=torch.uint8, device="cuda")
    else:
        store = torch.zeros((B, H, NB, lay["rec_bytes"]), dtype=torch.uint8, device="cuda")
    rows_k = torch.zeros((B, H, R, D), dtype=torch.float16, device="cuda")
    rows_v = torch.zeros_like(rows_k)
    # the new tokens lie as a layer's projections leave them: [batch, token, head, channel]
    q = torch.empty((B, n, Hq, D), dtype=dt, device="cuda")
    k = torch.empty((B, n, H, D), dtype=dt, device="cuda")
    v = torch.empty_like(k)
    for b in range(B):
        kc, qc = _outliers((H,), gen), _outliers((Hq,), gen)
        nb, r = counts[b][0] // lay["Rr"], counts[b][1]
        if nb:
            rec = _records(case, lay, kc, nb, gen)
            if table is not None:
                store[table[b, :nb].long()] = rec
            else:
                store[b, :, :nb] = rec.transpose(0, 1)
        for rows, c in ((rows_k, kc[:, None]), (rows_v, 1.0)):
            x = torch.randn((H, R, D), generator=gen, device="cuda") * _heavy_tail((H, R, 1), gen) * c
            rows[b, :, :r] = x.clamp(-32768.0, 32768.0)[:, :r]
        for new, c in ((k, kc), (v, 1.0)):
            x = torch.randn((n, H, D), generator=gen, device="cuda") * _heavy_tail((n, H, 1), gen) * c
            new[b] = x.clamp(-32768.0, 32768.0)
        q[b] = torch.randn((n, Hq, D), generator=gen, device="cuda") * qc
    state = dict(case=case, lay=lay, counts=counts, n_seq=n_seq, table=table, store=store, rows_k=rows_k, rows_v=rows_v,
                 q=q.transpose(1, 2), k=k.transpose(1, 2), v=v.transpose(1, 2),
                 out=torch.zeros((B, n, Hq, D), dtype=dt, device="cuda").transpose(1, 2))
    # what a program knows of its batch on the device
    state["n_packed"] = torch.tensor([c[0] for c in counts], device="cuda")
    state["n_rows"] = torch.tensor([c[1] for c in counts], device="cuda")
    state["n_new"] = torch.tensor(n_seq, device="cuda")
    if own:
        state["cache"] = _filled_cache(state, NB * lay["Rr"])
    return state


def _filled_cache(state, T_max):
    """The cache that a program would have filled by its appends, with the state's records and rows in it."""
    import paper_2512_19206_amd as M
    case, lay = state["case"], state["lay"]
    kw = dict(B=case["B"], Hq=case["hq"], Hkv=case["hkv"], D=D, T_max=T_max, Gk=lay["Gk"], Gv=lay["Gv"], R=case["R"],
              k4=case["k4"], k16=case["k16"], in_dtype=1 if case["dtype"] == "bf16" else 0)
    if case["thresholds"]:
        kw.update(policy=1, tau16=20.0, tau4=4.0)
    gc = M.Cache(M.make_config(**kw))
    gc.set_block_table(state["table"])
    for dst, src in ((gc.blocks, state["store"]), (gc.res_k, state["rows_k"]), (gc.res_v, state["rows_v"])):
        flat = src.view(torch.uint8).view(-1)
        dst[:flat.numel()] = flat
    for b, (nq, r) in enumerate(state["counts"]):
        gc.lib.mixkvq_cache_set_state_seq(gc.handle, b, nq, r, 0)
    return gc


def _prepare_verify(case, gen):
    B, n, V = case["B"], case["n"], case["V"]
    n_seq = _spread(case["n_min"], n, B)
    rand = lambda *shape: torch.rand(shape, generator=gen, device="cuda")
    logits = 2.5 * torch.randn((B, n + 1, V), generator=gen, device="cuda")
    p = torch.softmax(logits, dim=-1)
    near = logits[:, :n] + 0.7 * torch.randn((B, n, V), generator=gen, device="cuda")
    near = torch.softmax(near, dim=-1)
    # a looked-up draft is what the target finds likely about half of the time; a draft model's is drawn from its probabilities
    pick = near.view(-1, V) if not case["onehot"] else torch.where(rand(B, n, 1) < 0.5, near ** 3, near).view(-1, V)
    draft = (torch.log(pick) - torch.log(-torch.log(torch.rand(pick.shape, generator=gen, device="cuda").clamp(1e-20, 1 - 1e-7)))).argmax(-1)
    return dict(case=case, p=p, q=None if case["onehot"] else near, draft=draft.int().view(B, n).contiguous(), u=rand(B, n),
                u_next=rand(B), n_seq=torch.tensor(n_seq, dtype=torch.int32, device="cuda"),
                n_accepted=torch.zeros(B, dtype=torch.int32, device="cuda"),
                tokens=torch.zeros((B, n + 1), dtype=torch.int32, device="cuda"))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return _prepare_chunk(case, gen) if case["kind"] == "chunk" else _prepare_verify(case, gen)


# ---------------------------------------------------------------------------- one pass

def run(state):
    if own:
        import paper_2512_19206_amd as M
        if state["case"]["kind"] == "chunk":
            return M.mixkvq_chunk_attention(state["cache"], state["q"], state["k"], state["v"], n_seq=state["n_seq"], out=state["out"])[0]
        return M.mixkvq_verify_draft(state["p"], state["draft"], state["u"], state["u_next"], p_draft=state["q"], n_seq=state["n_seq"],
                                     n_accepted=state["n_accepted"], tokens=state["tokens"])
    return _plain_chunk(state) if state["case"]["kind"] == "chunk" else _plain_verify(state)


def _unpack(words, bits):
    """Packed codes along a new last axis: code i of a word in bits [16 (i & 1) + bits (i >> 1), + bits)."""
    i = torch.arange(32 // bits, device=words.device)
    return (words[..., None] >> (16 * (i & 1) + bits * (i >> 1)).int()) & ((1 << bits) - 1)


def _plain_keys(rec, lay):
    """Dequantized keys of records [..., rec_bytes]: fp32 [..., Rr, D]."""
    lead, Rr, Gk, NLp, k4, k16 = rec.shape[:-1], lay["Rr"], lay["Gk"], lay["NLp"], lay["k4"], lay["k16"]
    grouped = lambda name: _plane(rec, lay, name).float().repeat_interleave(Gk, dim=-2)      # scales of every token's group
    parts = [_unpack(_plane(rec, lay, "lo"), 2).view(lead + (Rr, NLp)) * grouped("lo_s") + grouped("lo_z")]
    if k4:
        parts.append(_unpack(_plane(rec, lay, "k4"), 4).view(lead + (Rr, k4)) * grouped("k4_s") + grouped("k4_z"))
    if k16:
        parts.append(_plane(rec, lay, "k16").float())
    # where channel d stands in [2 bit | 4 bit | fp16]: the listed ones by their entry, the others in ascending order
    idx = _plane(rec, lay, "idx").long()
    place = torch.arange(k16 + k4, device=rec.device)
    place = torch.where(place < k16, NLp + k4 + place, NLp + place - k16).expand(idx.shape)
    spot = torch.full(lead + (256,), -1, dtype=torch.long, device=rec.device).scatter_(-1, idx, place)[..., :D]
    low = spot < 0
    spot = torch.where(low, low.long().cumsum(-1) - 1, spot)
    return torch.gather(torch.cat(parts, dim=-1), -1, spot[..., None, :].expand(lead + (Rr, D)))


def _plain_values(rec, lay):
    lead, Rr = rec.shape[:-1], lay["Rr"]
    codes = _unpack(_plane(rec, lay, "v"), 2).transpose(-1, -2)                  # [..., Rr / 16, 16, D]
    if lay["interleave"]:      # code i of word w stands for token 64 (w / 4) + 8 (w % 4) + i % 8 + 32 (i / 8)
        codes = codes.reshape(lead + (Rr // 64, 4, 2, 8, D)).transpose(-4, -3)
    codes = codes.reshape(lead + (Rr, D))
    wide = lambda name: _plane(rec, lay, name).float().repeat_interleave(lay["Gv"], dim=-1)
    return codes * wide("v_s") + wide("v_z")


def _plain_chunk(state):
    case, lay, table = state["case"], state["lay"], state["table"]
    B, H, Hq, n = case["B"], case["hkv"], case["hq"], case["n"]
    rec = state["store"]
    if table is not None:
        rec = rec[table.long()].transpose(1, 2)                                 # [B, H, NB, rec_bytes]
    NB, Rr, R = rec.shape[2], lay["Rr"], case["R"]
    keep = lambda x: x.float().clamp(-65504.0, 65504.0).half().float()          # what the cache keeps of a tensor
    K = torch.cat([_plain_keys(rec, lay).view(B, H, NB * Rr, D), state["rows_k"].float(), keep(state["k"])], dim=2)
    # token t of [packed | window | new] can be seen by new token i of sequence b
    b1 = lambda name: state[name][:, None]
    at = lambda m: torch.arange(m, device=rec.device)[None]
    cached = torch.cat([at(NB * Rr) < b1("n_packed"), at(R) < b1("n_rows")], dim=1)[:, None].expand(B, n, NB * Rr + R)
    causal = (at(n)[0][:, None] >= at(n)[0][None])[None].expand(B, n, n)
    seen = torch.cat([cached, causal], dim=2)[:, None, None]                    # [B, 1, 1, n, T]
    q = keep(state["q"]).reshape(B, H, (Hq // H) * n, D)
    s = torch.matmul(q, K.transpose(2, 3)) * (1.0 / math.sqrt(D))
    del K
    s = s.view(B, H, Hq // H, n, -1).masked_fill_(~seen, -math.inf)
    s = torch.exp_(s.sub_(s.amax(dim=-1, keepdim=True)))
    total = s.sum(dim=-1, keepdim=True)
    V = torch.cat([_plain_values(rec, lay).view(B, H, NB * Rr, D), state["rows_v"].float(), keep(state["v"])], dim=2)
    o = torch.matmul(s.view(B, H, (Hq // H) * n, -1), V).view(B, H, Hq // H, n, D) / total
    rows = (at(n) < b1("n_new"))[:, None, :, None]
    return torch.where(rows, o.reshape(B, Hq, n, D).to(_dtype(case)), state["out"])


def _plain_verify(state):
    p, q, draft, B, n = state["p"], state["q"], state["draft"].long(), state["case"]["B"], state["case"]["n"]
    at = torch.arange(n + 1, device=p.device)
    pt = torch.gather(p[:, :n], 2, draft[..., None])[..., 0].double()
    qt = torch.gather(q, 2, draft[..., None])[..., 0].double() if q is not None else torch.ones_like(pt)
    ok = (state["u"].double() * qt < pt) & (at[:n] < state["n_seq"][:, None])
    stay = ok.long().cumprod(dim=1).sum(dim=1)
    row = torch.arange(B, device=p.device)
    w = p[row, stay].double()
    rejected = (stay < state["n_seq"])[:, None]
    last = stay.clamp(max=n - 1)
    if q is not None:
        less = q[row, last].double()
    else:      # all of a looked-up draft's probability is on its token
        less = torch.zeros_like(w).scatter_(1, draft[row, last][:, None], 1.0)
    rest = torch.where(rejected, (w - less).clamp(min=0.0), w)
    w = torch.where(rest.sum(dim=1, keepdim=True) > 0, rest, w)
    upto = w.cumsum(dim=1)
    following = (upto > state["u_next"].double()[:, None] * upto[:, -1:]).int().argmax(dim=1)
    tokens = torch.where(at < stay[:, None], torch.cat([draft, draft[:, :1]], dim=1), -1)
    tokens = torch.where(at == stay[:, None], following[:, None], tokens)
    return stay.int(), tokens.int()


# ---------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    if case["kind"] == "verify":      # one row of each kind of probabilities a sequence
        rows = 1 if case["onehot"] else 2
        return {"bytes": case["B"] * (4.0 * case["V"] * rows + 16 * case["n"]), "flops": 3.0 * case["B"] * case["V"]}
    lay, hq, hkv = _layout(case), case["hq"], case["hkv"]
    bytes_, flops = 0.0, 0.0
    for T, n in zip(*_lengths(case)):
        packed, rows = _counts(T, case["R"])
        if n == 0:
            continue
        bytes_ += hkv * (packed // lay["Rr"] * lay["rec_bytes"] + rows * 4 * D) + n * (2 * hkv + 2 * hq) * 2 * D
        flops += 4.0 * D * hq * (T * n + n * (n + 1) / 2)
    return {"bytes": bytes_, "flops": flops}


# ---------------------------------------------------------------------------- the definition in 64 bits

def _exact_codes(words, bits):
    """Codes [..., 32 / bits] of packed words by way of their half-words: even codes in the low one, odd in the high one."""
    half = words.contiguous().view(torch.int16).view(words.shape + (2,)).int() & 0xFFFF
    steps = [(half // (1 << (bits * j))) % (1 << bits) for j in range(16 // bits)]
    return torch.stack(steps, dim=-2).flatten(-2)


def _exact_block(rec, lay):
    """Keys and values of one KV head's records [nb, rec_bytes] in 64 bits, [nb * Rr, D] each."""
    nb, Rr, Gk, Gv = rec.shape[0], lay["Rr"], lay["Gk"], lay["Gv"]
    get = lambda name: _plane(rec, lay, name)
    idx = get("idx").cpu().numpy()
    keys = torch.zeros((nb, Rr, D), dtype=torch.float64, device="cuda")
    group = torch.arange(Rr, device="cuda") // Gk
    lo = _exact_codes(get("lo"), 2).flatten(-2).double() * get("lo_s").double()[:, group] + get("lo_z").double()[:, group]
    four = _exact_codes(get("k4"), 4).flatten(-2).double() * get("k4_s").double()[:, group] + get("k4_z").double()[:, group] if lay["k4"] else None
    raw = get("k16").double()
    kinds, first = np.unique(idx, axis=0, return_inverse=True)
    for m, chans in enumerate(kinds):            # records with the same lists of channels together
        at = torch.from_numpy(np.nonzero(first.reshape(-1) == m)[0]).cuda()
        tier16, tier4 = [int(c) for c in chans[:lay["k16"]] if c < D], [int(c) for c in chans[lay["k16"]:] if c < D]
        rest = [c for c in range(D) if c not in tier16 and c not in tier4]
        for src, to in ((lo, rest), (four, tier4), (raw, tier16)):
            if to:
                keys[at[:, None, None], torch.arange(Rr, device="cuda")[None, :, None], torch.tensor(to, device="cuda")] = src[at][..., :len(to)]
    codes = _exact_codes(get("v"), 2).double()
    values = torch.empty((nb, Rr, D), dtype=torch.float64, device="cuda")
    for w in range(Rr // 16):
        for i in range(16):
            t = 64 * (w // 4) + 8 * (w % 4) + i % 8 + 32 * (i // 8) if lay["interleave"] else 16 * w + i
            values[:, t] = codes[:, w, :, i]
    of = torch.arange(D, device="cuda") // Gv
    values = values * get("v_s").double()[..., of] + get("v_z").double()[..., of]
    return keys.view(nb * Rr, D), values.view(nb * Rr, D)


def _exact_chunk(state):
    case, lay = state["case"], state["lay"]
    H, g = case["hkv"], case["hq"] // case["hkv"]
    out = torch.zeros(state["out"].shape, dtype=torch.float64, device="cuda")
    most = np.float32(65504.0)
    kept = lambda x: torch.from_numpy(np.clip(x.float().cpu().numpy(), -most, most).astype(np.float16)).cuda().double()
    q, k, v = (kept(state[name]) for name in ("q", "k", "v"))
    for b, (packed, rows) in enumerate(state["counts"]):
        n, nb = state["n_seq"][b], packed // lay["Rr"]
        if n == 0:
            continue
        later = torch.ones((n, n), dtype=torch.bool, device="cuda").triu(1)
        for j in range(H):
            rec = state["store"][state["table"][b, :nb].long(), j] if state["table"] is not None else state["store"][b, j, :nb]
            K, V = [state["rows_k"][b, j, :rows].double(), k[b, j, :n]], [state["rows_v"][b, j, :rows].double(), v[b, j, :n]]
            if nb:
                kd, vd = _exact_block(rec, lay)
                K, V = [kd] + K, [vd] + V
            K, V = torch.cat(K), torch.cat(V)
            for h in range(j * g, (j + 1) * g):
                s = q[b, h, :n] @ K.T / math.sqrt(D)
                s[:, packed + rows:][later] = -math.inf
                out[b, h, :n] = torch.softmax(s, dim=-1) @ V
    return out


def _exact_verify(state):
    case = state["case"]
    stay, tokens = [], []
    draft, u, u_next, n_seq = (state[name].cpu().numpy() for name in ("draft", "u", "u_next", "n_seq"))
    for b in range(case["B"]):
        i = 0
        while i < n_seq[b]:
            t = int(draft[b, i])
            qt = float(state["q"][b, i, t]) if state["q"] is not None else 1.0
            if not float(u[b, i]) * qt < float(state["p"][b, i, t]):
                break
            i += 1
        w = state["p"][b, i].cpu().numpy().astype(np.float64)
        if i < n_seq[b]:
            if state["q"] is not None:
                rest = np.maximum(w - state["q"][b, i].cpu().numpy(), 0.0)
            else:
                rest = w.copy()
                rest[draft[b, i]] = 0.0
            w = rest if rest.sum() > 0 else w
        upto = np.cumsum(w)
        stay.append(i)
        tokens.append([int(t) for t in draft[b, :i]] + [int(np.searchsorted(upto, float(u_next[b]) * upto[-1], side="right"))] + [-1] * (case["n"] - i))
    return np.array(stay, dtype=np.int32), np.array(tokens, dtype=np.int32)


def exact(case, seed):
    state = prepare(case, seed)
    return _exact_chunk(state) if case["kind"] == "chunk" else _exact_verify(state)
