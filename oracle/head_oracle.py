"""CPU oracle for what stands between a block's last linear and the loss: the residual sum with the norms around it, token log
probabilities with entropy and top alternatives, and distillation from a teacher's listed entries, each with its gradient.

Test infrastructure only: plain numpy in fp64, row by row where that is plainer, no fusion, written from the definitions in
include/f8.h.  Inputs are fp64 arrays (of bf16 or fp32 values); results are unrounded, except that h of the residual sum can be
given as it is kept, since the norm after it reads the rounded values.  Pinned in tests/test_head_oracle_pins.py against
PyTorch's autograd in fp64, central differences and closed forms.
"""
import numpy as np


# ---- residual sum with the norms around it ------------------------------------------------

def _rstd(v, eps):
    return 1.0 / np.sqrt((v * v).mean(axis=1) + eps)


def _gate_rows(gate, M, D):
    return np.ones((M, D)) if gate is None else np.repeat(gate, M // gate.shape[0], axis=0)


def residual_h(x, y, g_post, gate, skip, branch, eps):
    """(h unrounded, rstd_post or None)"""
    r1 = None if g_post is None else _rstd(y, eps)
    u = y if g_post is None else y * r1[:, None] * g_post
    return skip * x + branch * _gate_rows(gate, *x.shape) * u, r1


def norm(h, g_pre, eps):
    r2 = _rstd(h, eps)
    return h * r2[:, None] * g_pre, r2


def _norm_grad(v, g, r, d):
    """(gradient of v, of g) of v * r(v) * g"""
    w = d * g
    return r[:, None] * w - v * (r ** 3 * (v * w).mean(axis=1))[:, None], (d * v * r[:, None]).sum(axis=0)


def residual_bwd(h, y, dh, dn, g_post, gate, g_pre, skip, branch, eps):
    """h: as kept.  dict of dx, dy, dg_post, dgate, dg_pre (those that exist)."""
    M, D = y.shape
    out = {}
    t = np.zeros((M, D)) if dh is None else dh
    if g_pre is not None:
        d, out["dg_pre"] = _norm_grad(h, g_pre, _rstd(h, eps), dn)
        t = t + d
    out["dx"] = skip * t
    r1 = None if g_post is None else _rstd(y, eps)
    u = y if g_post is None else y * r1[:, None] * g_post
    if gate is not None:
        out["dgate"] = (branch * t * u).reshape(gate.shape[0], -1, D).sum(axis=1)
    v = branch * _gate_rows(gate, M, D) * t
    if g_post is not None:
        v, out["dg_post"] = _norm_grad(y, g_post, r1, v)
    out["dy"] = v
    return out


# ---- logits -----------------------------------------------------------------------------------

def _softmax_row(z, scale):
    """(max, log sum exp(scale (z - max)), log p, p) of one row; -inf entries have p = 0, a row of nothing else p = 0 everywhere"""
    m = z.max()
    if m == -np.inf:
        return m, -np.inf, np.full_like(z, -np.inf), np.zeros_like(z)
    e = np.exp(scale * (z - m))
    s = e.sum()
    return m, np.log(s), scale * (z - m) - np.log(s), e / s


def token_logprobs(z, scale=1.0, targets=None, top_k=0):
    """dict of stats [M, 2], logp, entropy, top_ids, top_logp"""
    M, V = z.shape
    out = {"stats": np.zeros((M, 2)), "entropy": np.zeros(M), "logp": np.zeros(M), "top_ids": np.zeros((M, top_k), dtype=np.int64),
           "top_logp": np.zeros((M, top_k))}
    for r in range(M):
        m, ls, lp, p = _softmax_row(z[r], scale)
        out["stats"][r] = m, ls
        some = p > 0
        out["entropy"][r] = -(p[some] * lp[some]).sum()
        if targets is not None and targets[r] >= 0:
            out["logp"][r] = lp[targets[r]] if targets[r] < V else np.nan
        if top_k:
            ids = np.argsort(-z[r], kind="stable")[:top_k]
            out["top_ids"][r], out["top_logp"][r] = ids, lp[ids]
    return out


def token_logprobs_bwd(z, scale, targets, d_logp, d_entropy):
    M, V = z.shape
    dz = np.zeros((M, V))
    for r in range(M):
        m, ls, lp, p = _softmax_row(z[r], scale)
        if m == -np.inf:
            continue
        some = p > 0
        H = -(p[some] * lp[some]).sum()
        if d_entropy is not None:
            dz[r, some] -= d_entropy[r] * p[some] * (lp[some] + H)
        if d_logp is not None and targets[r] >= 0:
            dz[r] -= d_logp[r] * p
            dz[r, targets[r]] += d_logp[r]
    return scale * dz


def _teacher_row(ids, t, tail, teacher_scale):
    """(columns, q) of the entries that a row has"""
    there = (ids >= 0) & (t > -np.inf)
    ids, t = ids[there], t[there] * teacher_scale
    if len(ids) == 0:
        return ids, t
    return ids, np.exp(t) if tail else np.exp(t - t.max()) / np.exp(t - t.max()).sum()


def _has_term(ids, cols, tail):
    """whether a row has entries (tail), or weights to share out"""
    return (ids >= 0).any() if tail else len(cols) > 0


def _rest(listed, lp, q):
    """(q_rest, log p_rest, softmax outside the list): from the logs, so that a rest far below the list keeps its value"""
    q_rest, rest = 1.0 - q.sum(), lp[~listed]
    q_rest = 0.0 if q_rest < 2.0 ** -20 else q_rest
    top = rest.max() if rest.size else -np.inf
    if top == -np.inf:
        return q_rest, -np.inf, np.zeros_like(rest)
    e = np.exp(rest - top)
    return q_rest, top + np.log(e.sum()), e / e.sum()


def distill(z, ids, t, scale=1.0, tail=False, teacher_scale=1.0):
    """loss [M]"""
    M, V = z.shape
    loss = np.zeros(M)
    for r in range(M):
        _, _, lp, p = _softmax_row(z[r], scale)
        cols, q = _teacher_row(ids[r], t[r], tail, teacher_scale)
        if not _has_term(ids[r], cols, tail):
            continue
        loss[r] = sum(w * (np.log(w) - lp[c]) for c, w in zip(cols, q) if w > 0)
        if tail:
            listed = np.zeros(V, dtype=bool)
            listed[ids[r][ids[r] >= 0]] = True
            q_rest, log_rest, _ = _rest(listed, lp, q)
            if q_rest > 0:
                loss[r] += q_rest * (np.log(q_rest) - log_rest)
    return loss


def distill_bwd(z, ids, t, d_loss, scale=1.0, tail=False, teacher_scale=1.0, targets=None, d_logp=None):
    M, V = z.shape
    dz = np.zeros((M, V))
    for r in range(M):
        m, _, lp, p = _softmax_row(z[r], scale)
        if m == -np.inf:
            continue
        cols, q = _teacher_row(ids[r], t[r], tail, teacher_scale)
        listed = np.zeros(V, dtype=bool)
        listed[ids[r][ids[r] >= 0]] = True
        row = p.copy()
        if tail:
            q_rest, _, outside = _rest(listed, lp, q)
            row[~listed] -= q_rest * outside
        if _has_term(ids[r], cols, tail):
            np.add.at(row, cols, -q)
            dz[r] = d_loss[r] * row
        if targets is not None and targets[r] >= 0:
            dz[r] -= d_logp[r] * p
            dz[r, targets[r]] += d_logp[r]
    return scale * dz
