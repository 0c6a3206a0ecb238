"""Differential attention in 64 bits, from its definition, for the tests."""
import numpy as np


def reference(q, k, v, lam, lengths=None, causal=False, scale=None, do=None):
    """Arrays as the operator takes them (any float type; computed in float64).
    Returns o, or (o, dq, dk, dv, dlam) where `do` is given."""
    q, k, v, lam = (np.asarray(x, dtype=np.float64) for x in (q, k, v, lam))
    n, sq, hq, _, d = q.shape
    sk, hk, dv = k.shape[1], k.shape[2], v.shape[3]
    scale = d ** -0.5 if scale is None else scale
    per_head = np.broadcast_to(lam.reshape(-1), (hq,))
    o = np.zeros((n, sq, hq, dv))
    g = [np.zeros_like(x) for x in (q, k, v)] + [np.zeros(hq)]
    for b in range(n):
        length = sk if lengths is None else int(np.clip(lengths[b], 0, sk))
        for h in range(hq):
            kv = h // (hq // hk)
            for i in range(sq):
                seen = min(length, i + length - sq + 1) if causal else length
                if seen <= 0:
                    continue
                x = v[b, :seen, kv]
                maps = []
                for m in range(2):
                    s = scale * (k[b, :seen, kv, m] @ q[b, i, h, m])
                    e = np.exp(s - s.max())
                    maps.append(e / e.sum())
                w = maps[0] - per_head[h] * maps[1]
                o[b, i, h] = w @ x
                if do is None:
                    continue
                y = np.asarray(do, dtype=np.float64)[b, i, h]
                t = x @ y
                g[2][b, :seen, kv] += np.outer(w, y)
                g[3][h] -= maps[1] @ t
                for m, c in ((0, 1.0), (1, -per_head[h])):
                    ds = scale * c * maps[m] * (t - maps[m] @ t)
                    g[0][b, i, h, m] = ds @ k[b, :seen, kv, m]
                    g[1][b, :seen, kv, m] += np.outer(ds, q[b, i, h, m])
    if do is None:
        return o
    if lam.size == 1:
        g[3] = g[3].sum(keepdims=True)
    return (o, *g[:3], g[3].reshape(lam.shape))


def make_inputs(seed, n, sq, sk, hq, hk, d, dv, lam_count=None):
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    q, k, v, do = f(n, sq, hq, 2, d), f(n, sk, hk, 2, d), f(n, sk, hk, dv), f(n, sq, hq, dv)
    lam = rng.uniform(0.2, 0.8, lam_count or hq).astype(np.float32)
    return q, k, v, lam, do
