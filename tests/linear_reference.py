"""Linear attention in 64 bits, from its recurrence and from the adjoint
recurrence of it, token by token, for the tests."""
import numpy as np


def reference(q, k, v, log_decay, state=None, lengths=None, scale=None, do=None, dstate=None):
    """Arrays as the operator takes them (any float type; computed in float64).
    Returns (o, state), or (o, state, dq, dk, dv, gradient of the first state)
    where `do` is given."""
    q, k, v, log_decay = (np.asarray(x, dtype=np.float64) for x in (q, k, v, log_decay))
    n, s, hq, d = q.shape
    hk, dv = k.shape[2], v.shape[3]
    scale = d ** -0.5 if scale is None else scale
    group = hq // hk
    decay = np.exp(np.minimum(log_decay, 0.0))
    o, last = np.zeros((n, s, hq, dv)), np.zeros((n, hk, d, dv))
    dq, dk, dvalues, first = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v), np.zeros((n, hk, d, dv))
    for b in range(n):
        length = s if lengths is None else int(np.clip(lengths[b], 0, s))
        for g in range(hk):
            heads = slice(g * group, (g + 1) * group)
            x = np.zeros((d, dv)) if state is None else np.asarray(state[b, g], dtype=np.float64)
            states = []
            for t in range(length):
                x = decay[g] * x + np.outer(k[b, t, g], v[b, t, g])
                states.append(x)
                o[b, t, heads] = scale * q[b, t, heads] @ x
            last[b, g] = x
            if do is None:
                continue
            e = np.zeros((d, dv)) if dstate is None else np.asarray(dstate[b, g], dtype=np.float64)
            for t in range(length - 1, -1, -1):
                y = np.asarray(do[b, t, heads], dtype=np.float64)
                dq[b, t, heads] = scale * y @ states[t].T
                e = e + scale * q[b, t, heads].T @ y
                dk[b, t, g] = e @ v[b, t, g]
                dvalues[b, t, g] = e.T @ k[b, t, g]
                e = decay[g] * e
            first[b, g] = e
    return (o, last) if do is None else (o, last, dq, dk, dvalues, first)
