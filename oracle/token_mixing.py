"""fp64 CPU oracle for the norm of queries and keys with the rotary embedding, and for linear attention with a decay for
each KV head, forward and backward.

TEST INFRASTRUCTURE ONLY.  The plain definitions in NumPy float64, linear attention token by token; no code shared with the
GPU library, never imported by the product path.  `lengths` [B]: tokens of each batch row; the rest is padding, whose
outputs and gradients are zero.

Parity status: pinned by tests/test_oracle_token_mixing.py (closed forms, the sum over pairs, finite differences).
"""
from __future__ import annotations

import numpy as np

from oracle import decoder_layer as odl


def _lengths(lengths, batch, seq):
    return np.full(batch, seq) if lengths is None else np.clip(np.asarray(lengths), 0, seq)


def _angles(start, batch, seq, head_dim, base):
    """[B, S, dh/2]"""
    theta = np.power(np.float64(base), -2.0 * np.arange(head_dim // 2) / head_dim)
    first = np.zeros(batch) if start is None else np.asarray(start, dtype=np.float64)
    return (first[:, None] + np.arange(seq)[None])[..., None] * theta



def qk_norm_rope_fwd(x, gamma, eps, base, layout, start=None, lengths=None):
    """x [B, S, H, dh] (q or k), gamma [dh] -> (y [B, S, H, dh], rstd [B, S, H])."""
    B, S, _, dh = x.shape
    y, rstd = np.zeros(x.shape), np.zeros(x.shape[:-1])
    phi = _angles(start, B, S, dh, base)
    for b, n in enumerate(_lengths(lengths, B, S)):
        z, rstd[b, :n] = odl.rmsnorm_fwd(x[b, :n], gamma, eps)
        y[b, :n] = odl.rope_rotate(z[None], phi[b, :n], layout=layout)[0]
    return y, rstd


def qk_norm_rope_bwd(x, gamma, rstd, dy, base, layout, start=None, lengths=None):
    """Gradient of qk_norm_rope_fwd: (dx, dgamma)."""
    B, S, _, dh = x.shape
    dx, dgamma = np.zeros(x.shape), np.zeros(dh)
    phi = _angles(start, B, S, dh, base)
    for b, n in enumerate(_lengths(lengths, B, S)):
        dz = odl.rope_rotate(dy[None, b, :n], phi[b, :n], layout=layout, inverse=True)[0]
        dx[b, :n], dg = odl.rmsnorm_bwd(x[b, :n], gamma, rstd[b, :n], dz)
        dgamma += dg
    return dx, dgamma


def linear_attention_fwd(q, k, v, log_decay, scale, state=None, lengths=None):
    """q [B, S, Hq, dh], k, v [B, S, Hkv, dh], log_decay [Hkv], state [B, Hkv, dh, dh] -> (o [B, S, Hq, dh], state)."""
    B, S, Hq, dh = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    lam = np.exp(np.asarray(log_decay, np.float64))
    out_state = np.zeros((B, Hkv, dh, dh)) if state is None else np.array(state, np.float64)
    o = np.zeros(q.shape)
    for b, n in enumerate(_lengths(lengths, B, S)):
        s = out_state[b]
        for t in range(n):
            s = lam[:, None, None] * s + k[b, t, :, :, None] * v[b, t, :, None, :]
            o[b, t] = scale * np.einsum("jgd,jde->jge", q[b, t].reshape(Hkv, G, dh), s).reshape(Hq, dh)
        out_state[b] = s
    return o, out_state


def linear_attention_bwd(q, k, v, log_decay, scale, d_o, state=None, d_state_out=None, lengths=None):
    """Gradient of linear_attention_fwd: (dq, dk, dv, d_state_in)."""
    B, S, Hq, dh = q.shape
    Hkv = k.shape[2]
    G = Hq // Hkv
    lam = np.exp(np.asarray(log_decay, np.float64))[:, None, None]
    dq, dk, dv = np.zeros(q.shape), np.zeros(k.shape), np.zeros(v.shape)
    d_state = np.zeros((B, Hkv, dh, dh)) if d_state_out is None else np.array(d_state_out, np.float64)
    for b, n in enumerate(_lengths(lengths, B, S)):
        s = np.zeros((Hkv, dh, dh)) if state is None else np.asarray(state[b], np.float64)
        for t in range(n):
            s = lam * s + k[b, t, :, :, None] * v[b, t, :, None, :]
            dq[b, t] = scale * np.einsum("jde,jge->jgd", s, d_o[b, t].reshape(Hkv, G, dh)).reshape(Hq, dh)
        r = d_state[b]
        for t in reversed(range(n)):
            r = r + scale * np.einsum("jgd,jge->jde", q[b, t].reshape(Hkv, G, dh), d_o[b, t].reshape(Hkv, G, dh))
            dk[b, t] = np.einsum("jde,je->jd", r, v[b, t])
            dv[b, t] = np.einsum("jde,jd->je", r, k[b, t])
            r = lam * r
        d_state[b] = r
    return dq, dk, dv, d_state
