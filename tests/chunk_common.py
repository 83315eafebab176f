"""Reference of mixkvq_chunk_attention in 64 bits over an oracle cache's contents, with the bound that the kernel's roundings give
for every output."""
import numpy as np
import torch

from oracle import mixkvq_oracle as O

HALF = 2.0 ** -11        # half a step of binary16, relative


def kept(t: torch.Tensor) -> np.ndarray:
    """What the cache keeps of a tensor (binary16, saturated), in 64 bits."""
    if t.dtype == torch.bfloat16:
        return O.bf16_bits_to_f16(t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)).astype(np.float64)
    return t.cpu().numpy().astype(np.float64)


def chunk_reference(K0, V0, q, k, v, scale, out_half, key_size=None, rounds=None):
    """One KV head: K0, V0 [T, D] cached (64 bits), q [g, n, D], k, v [n, D].  Returns out [g, n, D], lse [g, n] and how far the
    kernel's may be from them.

    The weights are those of scores off by at most E_t: keys rounded to binary16 (half a step each, or 2^-25 below its normal
    range) and binary32 sums of 128 products.  With sum_t w_t (v_t - o) = 0 that moves the output by at most
    sum_t w_t (e^E_t - 1) |v_t - o| e^max(E).  Weights and values are rounded to binary16 (half a step each; a weight below
    2^-14 of the largest loses up to 2^-25), the sums over T tokens are binary32, the output is rounded once.  Where a token has
    one value group the kernel rounds p s instead of the value c s + z (Eq. 3): half a step of c s, which is the value less its
    group's smallest (that one has code 0); rounds [T, D]: what half a step is relative to, |values| unless given.
    key_size [T, D]: what half a step of binary16 is relative to in the scores, |keys| unless given.
    """
    g, n, D = q.shape
    T0 = K0.shape[0]
    K, V = np.concatenate([K0, k]), np.concatenate([V0, v])
    T = T0 + n
    s = np.einsum("gnd,td->gnt", q, K) * scale
    E = (np.einsum("gnd,td->gnt", np.abs(q), np.abs(K) if key_size is None else key_size) * (HALF + 130 * 2.0 ** -24) + np.abs(q).sum(-1)[..., None] * 2.0 ** -25) * scale
    E += np.abs(s) * 2.0 ** -22      # scale, reference and exponential in binary32
    seen = np.arange(T)[None] < T0 + 1 + np.arange(n)[:, None]
    s = np.where(seen, s, -np.inf)
    E = np.where(seen, E, 0.0)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(-1, keepdims=True)
    w = e / l
    o = w @ V
    Emax = E.max(-1, keepdims=True)
    up = np.exp(Emax)
    grow = w * np.expm1(E)
    # sum_t grow_t |v_t - o|, channel by channel
    err = np.stack([np.einsum("gnt,gntd->gnd", grow[:, i:i + 1], np.abs(V[None, None] - o[:, i:i + 1, None])) for i in range(n)], 1)[:, :, 0] * up
    size = w @ np.abs(V)
    err += up * (size * HALF + (size if rounds is None else w @ rounds) * (HALF + (T + 2) * 2.0 ** -24)) + np.abs(V).sum(0) * 2.0 ** -24
    err += out_half * (np.abs(o) + err) + 2.0 ** -25
    lse_err = Emax[..., 0] + (T + 4) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(m + np.log(l))[..., 0])
    return o, (m + np.log(l))[..., 0], err, lse_err


def value_rounds(oc, p, v):
    """What the values' rounding is relative to, [T, D] over the cached tokens and the new ones."""
    if oc.n_quant + oc.n_res + oc.n_sink == 0:
        return np.abs(v)
    V0 = oc.dequantized(p)[1]
    size = np.abs(np.concatenate([V0, v]))
    if oc.cfg.Gv == oc.cfg.D:
        size[:V0.shape[0]] += V0 - V0.min(axis=1, keepdims=True)      # (binary32 sums of both parts: their sizes add)
    return size


def check_chunk(oc_of, g, Hkv, q, k, v, n_seq, out, lse, scale=None, name=""):
    """oc_of(b) -> (oracle cache, first pair of sequence b in it)."""
    scale = scale or 1.0 / np.sqrt(128.0)
    qh, kh, vh = kept(q), kept(k), kept(v)
    got, got_lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
    out_half = torch.finfo(out.dtype).eps / 2
    worst = 0.0
    for b in range(q.shape[0]):
        n = n_seq[b]
        if n == 0:
            continue
        oc, p0 = oc_of(b)
        for j in range(Hkv):
            K0, V0 = oc.dequantized(p0 + j) if oc.n_quant + oc.n_res + oc.n_sink else (np.zeros((0, 128)),) * 2
            hs = slice(j * g, (j + 1) * g)
            o, l, err, lerr = chunk_reference(K0, V0, qh[b, hs, :n], kh[b, j, :n], vh[b, j, :n], scale, out_half,
                                              rounds=value_rounds(oc, p0 + j, vh[b, j, :n]))
            d = np.abs(got[b, hs, :n] - o)
            assert np.all(np.isfinite(got[b, hs, :n])), (name, b, j, "not finite")
            assert np.all(d <= err), (name, b, j, float((d / err).max()), float(d.max()))
            dl = np.abs(got_lse[b, hs, :n] - l)
            assert np.all(dl <= lerr), (name, b, j, "lse", float(dl.max()))
            worst = max(worst, float((d / err).max()))
    return worst
