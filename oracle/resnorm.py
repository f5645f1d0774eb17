"""The end of a block in 64 bits: norms before and after, gate, scaled residual; forward, and gradients by the chain rule."""
from __future__ import annotations

import numpy as np

NONE, LAYER, RMS = 0, 1, 2


def _hat(kind, v, eps):
    if kind == LAYER:
        v = v - v.mean(-1, keepdims=True)
    r = 1.0 / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    return v * r, r


def _affine(hat, gamma, beta):
    return hat * (1.0 if gamma is None else gamma) + (0.0 if beta is None else beta)


def _through(kind, g, hat, r):
    """dL/dv from g = dL/dhat."""
    mean = g.mean(-1, keepdims=True) if kind == LAYER else 0.0
    return r * (g - mean - hat * (g * hat).mean(-1, keepdims=True))


def gates_of_rows(gate, rows, rows_per_gate):
    if gate is None:
        return np.ones((1, 1))
    return gate.reshape(1, -1) if rows_per_gate == 0 else gate[np.arange(rows) // rows_per_gate]


def forward(x, b, gate, rows_per_gate, post, pre, params, scale, eps):
    """{h, y (None without a second norm), and what backward() reuses}; params = (post_gamma, post_beta, pre_gamma, pre_beta)."""
    pg, pb, qg, qb = params
    out = dict(gate=gates_of_rows(gate, x.shape[0], rows_per_gate), bhat=b, rb=None, hhat=None, rh=None, y=None)
    p = b
    if post != NONE:
        out["bhat"], out["rb"] = _hat(post, b, eps)
        p = _affine(out["bhat"], pg, pb)
    out["p"] = p
    out["h"] = scale * x + out["gate"] * p
    if pre != NONE:
        out["hhat"], out["rh"] = _hat(pre, out["h"], eps)
        out["y"] = _affine(out["hhat"], qg, qb)
    return out


def backward(f, dh, dy, rows_per_gate, post, pre, params, scale):
    """{dx, db, dgate, dpost_gamma, dpost_beta, dpre_gamma, dpre_beta} from forward()'s result."""
    pg, _, qg, _ = params
    d = np.zeros_like(f["h"]) if dh is None else dh
    out = {}
    if pre != NONE:
        out["dpre_gamma"], out["dpre_beta"] = (dy * f["hhat"]).sum(0), dy.sum(0)
        d = d + _through(pre, dy * (1.0 if qg is None else qg), f["hhat"], f["rh"])
    out["dx"] = scale * d
    t = d * f["p"]
    if rows_per_gate == 0:
        out["dgate"] = t.sum(0)
    else:
        out["dgate"] = np.add.reduceat(t, np.arange(0, t.shape[0], rows_per_gate), axis=0)
    dp = d * f["gate"]
    out["db"] = dp
    if post != NONE:
        out["dpost_gamma"], out["dpost_beta"] = (dp * f["bhat"]).sum(0), dp.sum(0)
        out["db"] = _through(post, dp * (1.0 if pg is None else pg), f["bhat"], f["rb"])
    return out
