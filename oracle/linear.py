"""CPU fp64 oracle of linear attention with a decay per head — TEST INFRASTRUCTURE ONLY.

The recurrence, token by token:  S = decay S + k v^T,  o = scale q^T S,  query head h reading state h // (Hq / Hkv).
"""
from __future__ import annotations

import numpy as np


def sequence(q, k, v, state, decay, scale):
    """q [n, Hq, d], k, v [n, Hkv, d], state [Hkv, d, d], all float64: (out [n, Hq, d], the state after the last token)."""
    G = q.shape[1] // k.shape[1]
    S = np.array(state, dtype=np.float64)
    lam = np.asarray(decay, dtype=np.float64)[:, None, None]
    out = np.empty(q.shape)
    for t in range(q.shape[0]):
        S = lam * S + k[t][:, :, None] * v[t][:, None, :]
        out[t] = scale * np.einsum("hgd,hde->hge", q[t].reshape(-1, G, q.shape[2]), S).reshape(q.shape[1:])
    return out, S


def chunks(q, k, v, states, decay, src, dst, cu, scale):
    """Ragged sequences over state slots: (out, the states afterwards)."""
    before, after = np.array(states, dtype=np.float64), np.array(states, dtype=np.float64)
    out = np.zeros(q.shape)
    for i in range(len(src)):
        a, b = int(cu[i]), int(cu[i + 1])
        S = before[src[i]] if src[i] >= 0 else np.zeros(before.shape[1:])
        out[a:b], S = sequence(q[a:b], k[a:b], v[a:b], S, decay, scale)
        if dst[i] >= 0:
            after[dst[i]] = S
    return out, after
