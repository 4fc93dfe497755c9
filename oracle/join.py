"""The gated, normed join of a branch into the residual stream, in float64:
out = alpha x + gate_s o RMSNorm(f; post), y = RMSNorm(out; pre), each of post,
gate and pre optional, and its gradients.  ``cu`` gives the rows of each sequence
where every sequence has a gate of its own ([n_seqs, h]); without it the gate, if
any, is one row.

TEST INFRASTRUCTURE ONLY.  Pinned by finite differences in the tests."""

from __future__ import annotations

import numpy as np


def _gate_rows(gate, cu, rows):
    if gate is None:
        return 1.0
    if cu is None:
        return np.asarray(gate, dtype=np.float64).reshape(1, -1)
    return np.repeat(gate, np.diff(cu), axis=0)[:rows]


def forward(x, f, post=None, gate=None, pre=None, cu=None, alpha=1.0, eps=1e-6):
    """dict of out, y, rstd_f, rstd_out (None where absent)."""
    rows = len(x)
    res = dict(y=None, rstd_f=None, rstd_out=None)
    n = f
    if post is not None:
        res["rstd_f"] = 1.0 / np.sqrt(np.mean(f * f, axis=1) + eps)
        n = f * res["rstd_f"][:, None] * post
    out = alpha * x + _gate_rows(gate, cu, rows) * n
    res["out"] = out
    if pre is not None:
        res["rstd_out"] = 1.0 / np.sqrt(np.mean(out * out, axis=1) + eps)
        res["y"] = out * res["rstd_out"][:, None] * pre
    return res


def backward(dout, dy, f, out, rstd_f, rstd_out, post=None, gate=None, pre=None, cu=None, alpha=1.0):
    """Gradients for <dout, out> + <dy, y> given the forward's f, out and row
    scales, and for each the sum of its terms' magnitudes (what rounding errors are
    relative to): two dicts with dx, df, y, dpost, dgate, dpre."""
    rows, h = dout.shape
    g, mag = {}, {}
    G, Gm = dout, np.abs(dout)
    if pre is not None:
        r = rstd_out[:, None]
        oh, d = out * r, pre * dy
        G = G + r * (d - oh * np.mean(d * oh, axis=1, keepdims=True))
        Gm = Gm + r * (np.abs(d) + np.abs(oh) * np.mean(np.abs(d * oh), axis=1, keepdims=True))
        g["dpre"], mag["dpre"] = np.sum(dy * oh, axis=0), np.sum(np.abs(dy * oh), axis=0)
        g["y"] = oh * pre
        mag["y"] = np.abs(g["y"])
    g["dx"], mag["dx"] = alpha * G, abs(alpha) * Gm
    rows_gate = _gate_rows(gate, cu, rows)
    dn, dnm = rows_gate * G, np.abs(rows_gate) * Gm
    if post is not None or gate is not None:
        fh = f if post is None else f * rstd_f[:, None]
        p = 1.0 if post is None else post
        if post is not None:
            g["dpost"], mag["dpost"] = np.sum(dn * fh, axis=0), np.sum(dnm * np.abs(fh), axis=0)
        if gate is not None:
            t, tm = G * fh * p, Gm * np.abs(fh * p)
            if cu is None:
                g["dgate"], mag["dgate"] = t.sum(axis=0), tm.sum(axis=0)
            else:
                add = lambda v: np.stack([v[a:b].sum(axis=0) for a, b in zip(cu[:-1], cu[1:])])
                g["dgate"], mag["dgate"] = add(t), add(tm)
        if post is not None:
            r, e, em = rstd_f[:, None], p * dn, np.abs(p) * dnm
            dn = r * (e - fh * np.mean(e * fh, axis=1, keepdims=True))
            dnm = r * (em + np.abs(fh) * np.mean(em * np.abs(fh), axis=1, keepdims=True))
    g["df"], mag["df"] = dn, dnm
    return g, mag
