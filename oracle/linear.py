"""fp64 CPU oracle for linear attention with a decay for each head (test infrastructure).

THIS IS TEST INFRASTRUCTURE: only the tests may import it; the GPU library never does and shares no code with it.

Per sequence and KV head, token by token as the definition has it, no chunks:
    S_t = e^(g_t) S_(t-1) + k_t v_t^T,   o_t = scale S_t^T q_t  for each query head of the group.
Gradients, with dS behind the last token given:
    dS_t = e^(g_(t+1)) dS_(t+1) + scale sum_h q_t do_t^T,   dq_t = scale S_t do_t,   dk_t = dS_t v_t,   dv_t = dS_t^T k_t,
    dg_t = e^(g_t) <S_(t-1), dS_t>,   dS_initial = e^(g_1) dS_1.
"""
from __future__ import annotations

import numpy as np


def _per_token(g, T, hkv):
    return np.broadcast_to(np.asarray(g, dtype=np.float64), (T, hkv))


def forward(q, k, v, g, lengths, scale, initial=None):
    """o [T, Hq, d] and the final states [B, Hkv, d, d]; g [T, Hkv] or [Hkv]; initial [B, Hkv, d, d] or None."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    g = _per_token(g, T, hkv)
    o, final = np.zeros(q.shape), np.zeros((len(lengths), hkv, d, d))
    t = 0
    for b, n in enumerate(lengths):
        S = np.zeros((hkv, d, d)) if initial is None else np.array(initial[b], dtype=np.float64)
        for _ in range(n):
            S = np.exp(g[t])[:, None, None] * S + k[t][:, :, None] * v[t][:, None, :]
            o[t] = scale * np.matmul(q[t].reshape(hkv, G, d), S).reshape(hq, d)
            t += 1
        final[b] = S
    return o, final


def backward(q, k, v, g, do, lengths, scale, initial=None, d_final=None):
    """dict of dq, dk, dv, dg [T, Hkv], d_initial [B, Hkv, d, d]."""
    T, hq, d = q.shape
    hkv = k.shape[1]
    G = hq // hkv
    g = _per_token(g, T, hkv)
    out = {"dq": np.zeros(q.shape), "dk": np.zeros(k.shape), "dv": np.zeros(k.shape), "dg": np.zeros((T, hkv)),
           "d_initial": np.zeros((len(lengths), hkv, d, d))}
    start = 0
    for b, n in enumerate(lengths):
        states = [np.zeros((hkv, d, d)) if initial is None else np.array(initial[b], dtype=np.float64)]
        for t in range(start, start + n):
            states.append(np.exp(g[t])[:, None, None] * states[-1] + k[t][:, :, None] * v[t][:, None, :])
        R = np.zeros((hkv, d, d)) if d_final is None else np.array(d_final[b], dtype=np.float64)
        for i in range(n, 0, -1):
            t = start + i - 1
            qs, ds = q[t].reshape(hkv, G, d), do[t].reshape(hkv, G, d)
            R = R + scale * np.matmul(qs.transpose(0, 2, 1), ds)
            out["dq"][t] = scale * np.matmul(ds, states[i].transpose(0, 2, 1)).reshape(hq, d)
            out["dk"][t] = np.matmul(R, v[t][:, :, None])[:, :, 0]
            out["dv"][t] = np.matmul(k[t][:, None, :], R)[:, 0]
            out["dg"][t] = np.exp(g[t]) * (states[i - 1] * R).sum((1, 2))
            R = np.exp(g[t])[:, None, None] * R
        out["d_initial"][b] = R
        start += n
    return out
