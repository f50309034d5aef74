"""float64 oracle of the gated-delta layer core, test infrastructure only: the equations of include/mamba_hip.h in a plain loop over
time (Yang, Kautz & Hatamizadeh, "Gated Delta Networks: Improving Mamba2 with Delta Rule", 2024), nothing chunked or reordered."""
import numpy as np

from .ssd import _silu, _softplus


def _sigmoid(v):
    return 1.0 / (1.0 + np.exp(-v))


def delta_scan(q, k, v, dt, A, beta, z=None, norm_w=None, dt_bias=None, h0=None, scale=None, eps=1e-6, dt_softplus=True,
               beta_sigmoid=True, qk_norm=True):
    """q, k (B,L,Hk,N); v, z (B,L,H,P); dt, beta (B,L,H); A, dt_bias (H); norm_w (P); h0 (B,H,P,N).
    Returns out (B,L,H,P) and the final state (B,H,P,N)."""
    q, k, v, dt, beta = (np.asarray(x, dtype=np.float64) for x in (q, k, v, dt, beta))
    B, L, H, P = v.shape
    Hk, N = q.shape[2:]
    scale = N ** -0.5 if scale is None else scale
    if qk_norm:
        q, k = (x / np.sqrt((x * x).sum(-1, keepdims=True) + eps) for x in (q, k))
    q, k = (np.repeat(x, H // Hk, axis=2) for x in (q, k))
    S = np.zeros((B, H, P, N)) if h0 is None else np.array(h0, dtype=np.float64)
    out = np.empty_like(v)
    for t in range(L):
        x = dt[:, t] + (0.0 if dt_bias is None else dt_bias)
        a = np.exp((_softplus(x) if dt_softplus else x) * A)[:, :, None, None]
        b = (_sigmoid(beta[:, t]) if beta_sigmoid else beta[:, t])[:, :, None]
        kt, qt = k[:, t], q[:, t]
        S = a * S
        u = b * (v[:, t] - (S * kt[:, :, None]).sum(-1))
        S = S + u[..., None] * kt[:, :, None]
        o = scale * (S * qt[:, :, None]).sum(-1)
        if norm_w is not None:
            o = o / np.sqrt((o * o).mean(-1, keepdims=True) + eps) * norm_w
        out[:, t] = o if z is None else o * _silu(np.asarray(z[:, t], dtype=np.float64))
    return out, S


def delta_step(h_in, q, k, v, dt, A, beta, z=None, norm_w=None, dt_bias=None, parent=None, **options):
    """One token for n_out branches; branch j continues from h_in[parent[j]].  Returns h_out, out."""
    src = np.asarray(h_in, dtype=np.float64)
    if parent is not None:
        src = src[np.asarray(parent)]
    one = lambda x: None if x is None else np.asarray(x)[:, None]
    out, S = delta_scan(one(q), one(k), one(v), one(dt), A, one(beta), one(z), norm_w, dt_bias, src, **options)
    return S, out[:, 0]
