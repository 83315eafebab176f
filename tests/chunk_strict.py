"""The formula of mixkvq_chunk_attention in 64 bits, with what every rounding of its kernels may move an output by: values (not their
parts) and weights to binary16, the keys too where many query rows share them."""
import numpy as np

HALF = 2.0 ** -11        # half a step of binary16, relative


def key_reach(K0, n_new):
    """What q.z and q.(c s) of Eq. 3 may be made of, [T + n_new, D] relative to |keys|: |z| + c s <= |key| + 2 range of the channel."""
    reach = np.zeros((K0.shape[0] + n_new, K0.shape[1]))
    if K0.shape[0]:
        reach[:K0.shape[0]] = 2 * np.ptp(K0, axis=0)
    return reach


def strict_reference(K0, V0, q, k, v, scale, out_half, rounded_keys, tail):
    """One KV head: K0, V0 [T, D] cached (64 bits), q [g, n, D], k, v [n, D].  Returns out, lse and how far the kernel's may be off.

    Scores: binary32 sums of 128 products and of their two parts, queries times scales to 22 bits, keys to 11 where rounded_keys.
    Weights are off by half a step of binary16 each or, where that is more, by `tail` of the row's largest one; so are their sums, from
    which nothing is rounded away again.  Values c s + z are off by half a step of their own, sums over T tokens are binary32, the
    output is rounded once."""
    g, n, D = q.shape
    T0 = K0.shape[0]
    K, V = np.concatenate([K0, k]), np.concatenate([V0, v])
    T = T0 + n
    s = np.matmul(q, K.T) * scale
    size = np.abs(K) * ((HALF if rounded_keys else 0.0) + 2.0 ** -21 + 130 * 2.0 ** -24) + key_reach(K0, n) * (2.0 ** -21 + 130 * 2.0 ** -24)
    E = (np.matmul(np.abs(q), size.T) + np.abs(q).sum(-1)[..., None] * 2.0 ** -25) * scale + np.abs(s) * 2.0 ** -22
    seen = np.arange(T)[None] < T0 + 1 + np.arange(n)[:, None]
    s, E = np.where(seen, s, -np.inf), np.where(seen, E, 0.0)
    m = s.max(-1, keepdims=True)
    e = np.exp(s - m)
    l = e.sum(-1, keepdims=True)
    w = e / l
    o = np.matmul(w, V)
    up = np.exp(E.max(-1, keepdims=True))
    # weights that are off by dw_t move the output by at most sum_t dw_t |v_t - o| (their sum takes them as they are)
    dw = (w * np.expm1(E) * up + (w * HALF + np.where(seen, tail, 0.0) / l)) * 1.01
    err = np.empty_like(o)
    for i in range(n):
        for h in range(g):
            err[h, i] = dw[h, i] @ np.abs(V - o[h, i])
    err += np.matmul(w, np.abs(V)) * (HALF + (T + 2) * 2.0 ** -24) * up + 2.0 ** -25
    err += out_half * (np.abs(o) + err) + 2.0 ** -25
    lse = (m + np.log(l))[..., 0]
    lse_err = E.max(-1) + HALF + (tail * seen.sum(-1) / l[..., 0]) + (T + 4) * 2.0 ** -24 + 2.0 ** -21 * (1 + np.abs(lse))
    return o, lse, err, lse_err
