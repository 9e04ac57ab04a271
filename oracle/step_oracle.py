"""CPU oracle for what a training step has around its blocks: token embeddings, layer norm, the norm of all gradients with its
clipping, each with its gradient where it has one.

Test infrastructure only: plain numpy in fp64, no fusion, written from the definitions in include/f8.h.  Inputs are fp64 arrays
(of bf16 or fp32 values); results are unrounded.  Pinned in tests/test_step_oracle_pins.py against PyTorch's autograd in fp64,
central differences and hand-worked cases.
"""
import numpy as np


# ---- token embeddings -------------------------------------------------------------------------

def embed(ids, table, scale):
    V, D = table.shape
    out = np.zeros((len(ids), D))
    for m, v in enumerate(ids):
        if v >= V:
            out[m] = np.nan
        elif v >= 0:
            out[m] = scale * table[v]
    return out


def embed_bwd(ids, dout, V, scale):
    """(the table's gradient, the sums of magnitudes that entered it, tokens of each id)"""
    d, mag, n = np.zeros((V, dout.shape[1])), np.zeros((V, dout.shape[1])), np.zeros(V, dtype=np.int64)
    for m, v in enumerate(ids):
        if 0 <= v < V:
            d[v] += dout[m]
            mag[v] += np.abs(dout[m])
            n[v] += 1
    return scale * d, abs(scale) * mag, n


# ---- layer norm -------------------------------------------------------------------------------

def layernorm(h, g, b, eps):
    """(n, mean, rstd) of h as it is kept; b may be None"""
    mean = h.mean(axis=1)
    c = h - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(axis=1) + eps)
    n = c * rstd[:, None] * g
    return (n if b is None else n + b), mean, rstd


def layernorm_bwd(h, g, dn, dh, eps):
    """(dx, dg, db); dh may be None"""
    _, mean, rstd = layernorm(h, g, None, eps)
    c = (h - mean[:, None]) * rstd[:, None]
    v = g * dn
    dx = rstd[:, None] * (v - v.mean(axis=1, keepdims=True) - c * (v * c).mean(axis=1, keepdims=True))
    return (dx if dh is None else dx + dh), (dn * c).sum(axis=0), dn.sum(axis=0)


# ---- the norm of all gradients ------------------------------------------------------------------

def grad_norm(tensors, largest=False):
    """(norm, sum): sum of squares or largest magnitude; NaN if there is a NaN"""
    if largest:
        parts = [np.abs(t).max() for t in tensors if t.size]
        m = float(np.max(parts)) if parts else 0.0   # (numpy's maxima keep a NaN)
        return m, m
    s = float(sum((t * t).sum() for t in tensors))
    return np.sqrt(s), s


def clip_factor(norm, most):
    """In fp32, as the definition has it: min(1, most / (norm + 1e-6))"""
    with np.errstate(divide="ignore", invalid="ignore", over="ignore"):
        f = np.float32(most) / (np.float32(norm) + np.float32(1e-6))
    return np.float32(1.0) if f > 1 else f
