"""Float64 oracle of the transformer block: the layer with gated, normed joins,
y1 = rms(x) norm1, q, k, v = y1 W, o = attention, (h, y2) = join of o Wo into x
(post1, gate1, norm2), u = y2 Wup, out = join of gelu(u) Wdown into h (post2,
gate2); and its backward from kept activations, which may be those that a stash of
fewer bits holds.

TEST INFRASTRUCTURE ONLY.  The gradients from the forward's own activations are
pinned by finite differences in the tests.
"""

from __future__ import annotations

import numpy as np

from oracle import attention as A
from oracle import join as J
from oracle import layer as LY


def _join(W, i, cu):
    w = dict(post=W.get(f"post{i}"), gate=W.get(f"gate{i}"))
    per = w["gate"] is not None and np.ndim(w["gate"]) == 2 and len(w["gate"]) > 1
    return w, (np.asarray(cu) if per else None)


def forward(x, W, cu, H, D, scale, causal, eps, alpha):
    """(out, kept): kept holds what the backward needs, unrounded."""
    T = len(x)
    y1, _ = LY.rmsnorm(x, W["norm1"], eps)
    q, k, v = (y1 @ W[n] for n in ("wq", "wk", "wv"))
    o, lse = A.attention_forward(q.reshape(T, H, D), k.reshape(T, H, D), v.reshape(T, H, D), cu, scale, causal)
    o = o.reshape(T, H * D)
    f1 = o @ W["wo"]
    w, per = _join(W, 1, cu)
    j1 = J.forward(x, f1, pre=W["norm2"], cu=per, alpha=alpha, eps=eps, **w)
    u = j1["y"] @ W["w_up"]
    f2 = LY.gelu(u) @ W["w_down"]
    w, per = _join(W, 2, cu)
    j2 = J.forward(j1["out"], f2, cu=per, alpha=alpha, eps=eps, **w)
    kept = dict(q=q, k=k, v=v, o=o, f1=f1, h=j1["out"], u=u, f2=f2, lse=lse, rstd_f1=j1["rstd_f"],
                rstd_h=j1["rstd_out"], rstd_f2=j2["rstd_f"])
    return j2["out"], kept


def backward(dout, x, W, K, cu, H, D, scale, causal, eps, alpha):
    """(dx, gradients by name) from the kept activations K."""
    T, h = x.shape
    g = {}
    w, per = _join(W, 2, cu)
    j2, _ = J.backward(dout, None, K["f2"], None, K["rstd_f2"], None, cu=per, alpha=alpha, **w)
    da = j2["df"] @ W["w_down"].T
    g["w_down"] = LY.gelu(K["u"]).T @ j2["df"]
    du = da * LY.gelu_grad(K["u"])
    w, per = _join(W, 1, cu)
    j1, _ = J.backward(j2["dx"], du @ W["w_up"].T, K["f1"], K["h"], K["rstd_f1"], K["rstd_h"], pre=W["norm2"],
                       cu=per, alpha=alpha, **w)
    g["w_up"] = j1["y"].T @ du
    g["norm2"] = j1["dpre"]
    for i, j in ((1, j1), (2, j2)):
        if f"post{i}" in W:
            g[f"post{i}"] = j["dpost"]
        if f"gate{i}" in W:
            g[f"gate{i}"] = j["dgate"].reshape(np.shape(W[f"gate{i}"]))
    df1 = j1["df"]
    g["wo"] = K["o"].T @ df1
    heads = lambda a: a.reshape(T, H, D)
    dq, dk, dv = attention_backward(heads(df1 @ W["wo"].T), heads(K["q"]), heads(K["k"]), heads(K["v"]), heads(K["o"]),
                                    K["lse"], cu, scale, causal)
    y1, r1 = LY.rmsnorm(x, W["norm1"], eps)
    dy1 = 0.0
    for n, d in (("wq", dq), ("wk", dk), ("wv", dv)):
        d = d.reshape(T, h)
        g[n] = y1.T @ d
        dy1 = dy1 + d @ W[n].T
    dz, g["norm1"] = LY.rmsnorm_backward(dy1, x, W["norm1"], r1)
    return j1["dx"] + dz, g


def attention_backward(do, q, k, v, o, lse, cu, scale, causal):
    """Gradients with P = exp(scale Q K^T - lse) for the given lse [H, T] and rowsum(dO
    o O) for the given o: what a backward from kept activations computes."""
    dq, dk, dv = np.zeros_like(q), np.zeros_like(k), np.zeros_like(v)
    for lo, hi in zip(cu[:-1], cu[1:]):
        for n in range(q.shape[1]):
            Q, Kn, V, dO = (a[lo:hi, n] for a in (q, k, v, do))
            S = scale * Q @ Kn.T
            if causal:
                S = np.where(np.tril(np.ones(S.shape, dtype=bool)), S, -np.inf)
            P = np.exp(S - lse[n, lo:hi, None])
            dS = P * (dO @ V.T - np.sum(dO * o[lo:hi, n], axis=1, keepdims=True))
            dq[lo:hi, n], dk[lo:hi, n], dv[lo:hi, n] = scale * dS @ Kn, scale * dS.T @ Q, P.T @ dO
    return dq, dk, dv
