"""Linear attention with a decay for each head in fp64, token by token.

Test infrastructure only (see the package docstring). The recurrence as it is
written: for every sequence and query head a state S [Dk][Dv],

    S_t = exp(g) S_(t-1) + k_t v_t^T,   o_t = scale S_t^T q_t,

and its adjoint,

    dq_t = scale S_t dO_t,  G_t = exp(g) G_(t+1) + scale q_t dO_t^T,
    dk_t = G_t v_t,  dv_t = G_t^T k_t,

with the gradient of the last state in the place of exp(g) G_(length) and
ds0 = exp(g) G_0. Tensors are [B][T][heads][width]; query heads that share a
key head add their gradients up.
"""
import numpy as np


def _shared(x, heads):
    return np.repeat(x, heads // x.shape[2], axis=2)


def forward(q, k, v, log_decay, lengths=None, s0=None, scale=1.0):
    """(o, sT, states after each token [T] of [B][H][Dk][Dv]); tokens from a
    sequence's length on give zeros and leave its state."""
    q, k, v = (np.asarray(a, np.float64) for a in (q, k, v))
    B, T, H, Dk = q.shape
    k, v = _shared(k, H), _shared(v, H)
    decay = np.exp(np.asarray(log_decay, np.float64))[None, :, None, None]
    S = np.zeros((B, H, Dk, v.shape[3])) if s0 is None else np.array(s0, np.float64)
    o, states = np.zeros((B, T, H, v.shape[3])), []
    for t in range(T):
        on = np.ones(B, bool) if lengths is None else t < np.asarray(lengths)
        S = S.copy()
        S[on] = (S * decay if t or s0 is not None else S)[on] + np.einsum("bhm,bhn->bhmn", k[on, t], v[on, t])
        o[on, t] = scale * np.einsum("bhm,bhmn->bhn", q[on, t], S[on])
        states.append(S)
    return o, S, states


def backward(q, k, v, do, log_decay, lengths=None, s0=None, dsT=None, scale=1.0):
    """(dq, dk, dv, ds0)."""
    q, k, v, do = (np.asarray(a, np.float64) for a in (q, k, v, do))
    B, T, H, Dk = q.shape
    Hk, Dv = k.shape[2], v.shape[3]
    _, _, states = forward(q, k, v, log_decay, lengths, s0, scale)
    k, v = _shared(k, H), _shared(v, H)
    decay = np.exp(np.asarray(log_decay, np.float64))[None, :, None, None]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    G = np.zeros((B, H, Dk, Dv)) if dsT is None else np.array(dsT, np.float64)
    for t in range(T - 1, -1, -1):
        on = np.ones(B, bool) if lengths is None else t < np.asarray(lengths)
        dq[on, t] = scale * np.einsum("bhmn,bhn->bhm", states[t][on], do[on, t])
        here = G[on] + scale * np.einsum("bhm,bhn->bhmn", q[on, t], do[on, t])
        dk[on, t] = np.einsum("bhmn,bhn->bhm", here, v[on, t])
        dv[on, t] = np.einsum("bhmn,bhm->bhn", here, k[on, t])
        G[on] = here * decay
    add = lambda x: x.reshape(B, T, Hk, H // Hk, -1).sum(axis=3)
    return dq, add(dk), add(dv), G
