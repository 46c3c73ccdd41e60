"""TEST INFRASTRUCTURE: gradients of the gated delta rule in fp64, token by token.

With a = exp(g):  e = v - a k S,  S <- a S + beta k' e,  o = scale q S  (App. A.1, Eq. 11-12; output rule Eq. 3), differentiated
step by step from the last token to the first.  Shares no code with the GPU path.
"""
import numpy as np


def forward(S, q, k, v, g, beta, scale):
    """One sequence: S [Hv,dk,dv], q, k [T,Hk,dk], v [T,Hv,dv], g, beta [T,Hv].  Returns (o [T,Hv,dv], states before each token, S)."""
    r = v.shape[1] // q.shape[1]
    before, out = [], np.zeros(v.shape)
    for t in range(len(q)):
        kt, qt, a = np.repeat(k[t], r, 0), np.repeat(q[t], r, 0), np.exp(g[t])[:, None]
        before.append(S)
        e = v[t] - a * np.einsum("hk,hkv->hv", kt, S)
        S = a[:, :, None] * S + kt[:, :, None] * (beta[t][:, None] * e)[:, None, :]
        out[t] = scale * np.einsum("hk,hkv->hv", qt, S)
    return out, before, S


def backward(S0, q, k, v, g, beta, scale, dout, dS):
    """Gradients (dq, dk, dv, dg, dbeta, dS0) of <out, dout> + <last state, dS> for one sequence, all fp64."""
    S0, q, k, v, g, beta, dout, dS = (np.asarray(x, np.float64) for x in (S0, q, k, v, g, beta, dout, dS))
    r = v.shape[1] // q.shape[1]
    _, before, S = forward(S0, q, k, v, g, beta, scale)
    dq, dk, dv, dg, dbeta = (np.zeros(x.shape) for x in (q, k, v, g, beta))
    for t in reversed(range(len(q))):
        kt, qt, a, P = np.repeat(k[t], r, 0), np.repeat(q[t], r, 0), np.exp(g[t])[:, None], before[t]
        kP = np.einsum("hk,hkv->hv", kt, P)
        e = v[t] - a * kP
        do = scale * dout[t]
        dS = dS + qt[:, :, None] * do[:, None, :]
        du = np.einsum("hk,hkv->hv", kt, dS)
        de = beta[t][:, None] * du
        dbeta[t] = (du * e).sum(-1)
        dv[t] = de
        dq[t] = np.einsum("hkv,hv->hk", S, do).reshape(-1, r, q.shape[2]).sum(1)
        dk[t] = (np.einsum("hkv,hv->hk", dS, beta[t][:, None] * e) - a * np.einsum("hkv,hv->hk", P, de)).reshape(-1, r, k.shape[2]).sum(1)
        dg[t] = a[:, 0] * ((dS * P).sum((1, 2)) - (kP * de).sum(-1))
        dS = a[:, :, None] * (dS - kt[:, :, None] * de[:, None, :])
        S = P
    return dq, dk, dv, dg, dbeta, dS
