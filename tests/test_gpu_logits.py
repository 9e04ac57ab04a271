"""f8.token_logprobs, f8.distill and their backwards through the C ABI against oracle/head_oracle.py (fp64).

Tolerances, with z = scale * logits, l = log p and u = 2^-24 (half a step of fp32).  The exponent (z_j - z_max) log2(e) is off by
at most 4 u of itself (the difference, the constant, its product with the scale, their product), the exponential itself by 4 u, and
a sum over V terms takes at most V / 512 / blocks + 40 additions one after the other.  So the log of the sum is off by
  dl = 4 u sum_j p_j |z_j - z_max| + (V / 512 + 48) u + 2 u |log sum|
and every p_j by a factor within 4 u |z_j - z_max| + dl + 8 u.  bf16 results add half a step, 2^-8 of the value."""
import numpy as np
import pytest
import torch

import oracle as o
from oracle import head_oracle as ho
from paper_2410_06511_amd import f8
from helpers import bits

pytestmark = pytest.mark.gpu

HALF, U = 2.0 ** -8, 2.0 ** -24
LOWEST = -3.3895313892515355e38  # bf16's


def wide(t):
    return o.bf16_to_f32(bits(t)).astype(np.float64)


def f64(t):
    return t.cpu().numpy().astype(np.float64)


def make_logits(M, V, seed, std=3.0, cols=None, pitch=0):
    """[M, cols] on the GPU (cols: V rounded up to 16), `pitch` more columns between rows; what is beyond V is NaN."""
    cols = cols or (V + 15) // 16 * 16
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    t = torch.full((M, cols + pitch), float("nan"), dtype=torch.bfloat16, device="cuda")
    t[:, :V] = (torch.randn((M, V), generator=g) * std).to(torch.bfloat16).cuda()
    return t[:, :cols]


def make_targets(M, V, seed):
    t = torch.from_numpy(np.random.default_rng(seed).integers(0, V, M))
    t[::7] = -1
    if M > 1:
        t[1] = V - 1
    return t.cuda()


def forward(z, V, scale=1.0, targets=None, k=0, entropy=True, stream=None):
    M = z.shape[0]
    f32 = lambda *s: torch.full(s, 77.0, device="cuda")
    r = dict(stats=f32(M, 2), logp=f32(M) if targets is not None else None, entropy=f32(M) if entropy else None,
             top_ids=torch.full((M, k), -7, dtype=torch.int64, device="cuda") if k else None, top_logp=f32(M, k) if k else None)
    ws = torch.full((f8.logits_workspace_bytes(M, V, k),), 255, dtype=torch.uint8, device="cuda")
    f8.token_logprobs(z, V, r["stats"], targets, r["logp"], r["entropy"], r["top_ids"], r["top_logp"], scale, ws, stream)
    return r


def errors(zw, scale):
    """(dl a row, factor of every p) as derived above, for rows with something left"""
    M, V = zw.shape
    with np.errstate(invalid="ignore", over="ignore"):
        m = zw.max(axis=1, keepdims=True)
        d = np.where(np.isfinite(m) & (zw > -np.inf), scale * (m - zw), 0.0)
        p = np.where(zw > -np.inf, np.exp(-np.minimum(d, 800)), 0.0)
        s = np.maximum(p.sum(axis=1, keepdims=True), 1e-300)
    dl = (4 * U * (p / s * d).sum(axis=1) + (V / 512 + 48) * U + 2 * U * np.abs(np.log(s[:, 0])))
    return dl, 4 * U * np.minimum(d, 800) + dl[:, None] + 8 * U, p / s, d + np.log(s)


def check_forward(z, V, r, scale, targets, k):
    zw = wide(z)[:, :V]
    M = zw.shape[0]
    t = None if targets is None else targets.cpu().numpy()
    ref = ho.token_logprobs(zw, scale, t, k)
    dl, fp, p, nl = errors(zw, scale)
    got = f64(r["stats"])
    assert np.array_equal(got[:, 0], ref["stats"][:, 0])
    some = ref["stats"][:, 1] > -np.inf
    assert np.array_equal(got[~some, 1], ref["stats"][~some, 1])
    assert (np.abs(got[some, 1] - ref["stats"][some, 1]) <= dl[some]).all()

    def logs_close(got, ref, dl):
        # between the type's lowest and largest value lie 6.8e38, twice fp32's largest: the nearest fp32 value is -inf
        with np.errstate(over="ignore"):
            dead = ref.astype(np.float32) == -np.inf
        assert np.array_equal(got == -np.inf, dead)
        assert (np.abs(got[~dead] - ref[~dead]) <= np.broadcast_to(dl, got.shape)[~dead] + 6 * U * np.abs(ref[~dead])).all()
    if t is not None:
        # (z_t - z_max) scale = logp + log sum, each rounded: 6 U of logp and, within dl, 2 U of the log
        logs_close(f64(r["logp"]), ref["logp"], 2 * dl)
    if r["entropy"] is not None:
        dh = 2 * dl + (p * nl * (fp + 4 * U)).sum(axis=1) + 8 * U * ref["entropy"] + (V / 512 + 48) * U * (p * nl).sum(axis=1)
        assert (np.abs(f64(r["entropy"]) - ref["entropy"]) <= dh).all()
    if k:
        assert np.array_equal(r["top_ids"].cpu().numpy(), ref["top_ids"])
        logs_close(f64(r["top_logp"]), ref["top_logp"], 2 * dl[:, None])
    return ref


def backward(z, V, r, scale, targets, d_logp, d_entropy, cols=None, out=None, amax=True, stream=None):
    M = z.shape[0]
    dz = out if out is not None else torch.full((M, cols or z.shape[1]), 9.0, dtype=torch.bfloat16, device="cuda")
    am = torch.full((1,), -1.0, device="cuda") if amax else None
    f8.token_logprobs_bwd(z, V, r["stats"], dz, targets, r["entropy"] if d_entropy is not None else None, d_logp, d_entropy, scale, am,
                          f8.new_workspace(1, 1), stream)
    return dz, am


def check_gradient(zw, V, dz, am, ref, scale, weight, dh_weight=None):
    """weight: the sum of the magnitudes that multiply p_j in each element, per row; dh_weight: |d_entropy| a row"""
    got = wide(dz)
    assert not got[:, V:].any()
    _, fp, p, nl = errors(zw, scale)
    mag = p * weight[:, None]
    bound = HALF * np.abs(ref) + scale * mag * (fp + 16 * U)
    if dh_weight is not None:
        H = (p * nl).sum(axis=1, keepdims=True)
        # the log of p_j is off by the factor of p_j, the entropy by as much in the mean
        bound += scale * p * dh_weight[:, None] * ((nl + H) * (fp + 16 * U) + 2 * fp + 2 * (p * (fp + 16 * U) * (1 + nl)).sum(axis=1, keepdims=True)
                                                   + (V / 512 + 48) * U * H)
    bad = np.abs(got[:, :V] - ref) > bound + 1e-38
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])
    if am is not None:
        assert am.item() == np.abs(got).max(initial=0.0)


# vocabularies below, at and above what a thread, a block and a row's pieces take; odd ones; few rows (shared by blocks) and many
SIZES = [(1, 1, 1), (2, 7, 3), (5, 8, 8), (3, 100, 20), (9, 513, 5), (4, 4099, 64), (2, 20000, 128), (1, 50001, 20), (70, 9001, 32), (600, 1000, 1),
         (3, 131072, 128), (520, 8192, 10), (2, 300007, 50)]


@pytest.mark.parametrize("M,V,k", SIZES)
@pytest.mark.parametrize("scale", (1.0, 0.3))
def test_logprobs_against_the_oracle(M, V, k, scale):
    z = make_logits(M, V, M + V)
    targets = make_targets(M, V, V)
    r = forward(z, V, scale, targets, k)
    torch.cuda.synchronize()
    check_forward(z, V, r, scale, targets, k)
    g = torch.Generator("cpu")
    g.manual_seed(V)
    d_logp, d_entropy = torch.randn(M, generator=g).cuda(), torch.randn(M, generator=g).cuda()
    zw, t = wide(z)[:, :V], targets.cpu().numpy()
    wl, wh = np.abs(f64(d_logp)) * (t >= 0), np.abs(f64(d_entropy))
    for dlp, dh in ((d_logp, None), (d_logp, d_entropy), (None, d_entropy)):
        tt = targets if dlp is not None else None
        dz, am = backward(z, V, r, scale, tt, dlp, dh)
        torch.cuda.synchronize()
        ref = ho.token_logprobs_bwd(zw, scale, t, None if dlp is None else f64(dlp), None if dh is None else f64(dh))
        check_gradient(zw, V, dz, am, ref, scale, wl if dlp is not None else 0 * wl, wh if dh is not None else None)


def test_outputs_do_not_depend_on_which_are_asked_for():
    M, V = 6, 70000
    z, targets = make_logits(M, V, 1), make_targets(M, V, 1)
    full = forward(z, V, 1.0, targets, 16)
    for entropy in (False, True):
        for k in (0, 3, 16):
            r = forward(z, V, 1.0, targets, k, entropy)
            assert torch.equal(r["stats"], full["stats"]) and torch.equal(r["logp"], full["logp"])
            if entropy:
                assert torch.equal(r["entropy"], full["entropy"])
            if k:
                assert torch.equal(r["top_ids"], full["top_ids"][:, :k]) and torch.equal(r["top_logp"], full["top_logp"][:, :k])
    alone = forward(z, V)
    assert torch.equal(alone["stats"], full["stats"])


def special_rows(V):
    g = np.random.default_rng(V)
    rows = {
        "one value": np.full(V, 1.5),
        "both zeros": np.where(g.random(V) < 0.5, 0.0, -0.0),
        "nothing left": np.full(V, -np.inf),
        "one left": np.where(np.arange(V) == V // 2, -2.0, -np.inf),
        "a few left": np.where(np.arange(V) % 997 == 3, g.normal(size=V), -np.inf),
        "a stretch left": np.where((np.arange(V) > V // 3) & (np.arange(V) < V // 3 + 300), g.normal(size=V), -np.inf),
        "all lowest": np.full(V, LOWEST),
        "lowest as a mask": np.where(np.arange(V) % 3 == 0, g.normal(size=V), LOWEST),
        "lowest and -inf": np.where(np.arange(V) % 2 == 0, LOWEST, -np.inf),
        "largest": np.where(np.arange(V) == 5, -LOWEST, LOWEST),
        "far above": 1000.0 + g.normal(size=V),
        "ascending": np.linspace(-8, 8, V),
        "descending": np.linspace(8, -8, V),
        "large ones a block's threads apart": np.where(np.arange(V) // 8 % 512 < 3, 5 + g.random(V), g.normal(size=V) * 0.01),
        "every element of some threads": np.where(np.arange(V) // 8 % 512 < 60, 5 + g.random(V), -1.0),
        "few values": np.round(g.normal(size=V)),
    }
    return list(rows), np.stack(list(rows.values()))


# rows shared by blocks (few), and a row a block (many copies), with a length that no chunk divides
@pytest.mark.parametrize("V,copies,k", [(41, 1, 20), (5003, 1, 128), (5003, 40, 64), (100003, 1, 100), (100003, 40, 128)])
def test_masked_tied_and_ordered_rows(V, copies, k):
    names, rows = special_rows(V)
    n = len(names)
    z = torch.full((n * copies, (V + 15) // 16 * 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    z[:, :V] = torch.from_numpy(np.tile(rows, (copies, 1)).astype(np.float32)).to(torch.bfloat16).cuda()
    targets = torch.full((n * copies,), V // 2, dtype=torch.int64, device="cuda")
    r = forward(z, V, 1.0, targets, k)
    first = {key: v[:n] for key, v in r.items()}
    for key, v in r.items():  # every copy alike
        assert torch.equal(v, first[key].repeat((copies,) + (1,) * (v.dim() - 1))), key
    check_forward(z[:n], V, first, 1.0, targets[:n], k)
    d = torch.ones(n * copies, device="cuda")
    dz, am = backward(z, V, r, 1.0, targets, d, 0.5 * d)
    torch.cuda.synchronize()
    zw = wide(z[:n])[:, :V]
    ref = ho.token_logprobs_bwd(zw, 1.0, targets[:n].cpu().numpy(), np.ones(n), 0.5 * np.ones(n))
    assert torch.equal(dz.view(torch.int16), dz[:n].repeat(copies, 1).view(torch.int16))
    check_gradient(zw, V, dz[:n], am, ref, 1.0, np.ones(n), 0.5 * np.ones(n))


@pytest.mark.parametrize("M", (3, 600))
def test_rows_with_nan_or_infinity_are_nan_and_stay_alone(M):
    V, k = 9000, 40
    z = make_logits(M, V, 5)
    z[0, 17], z[2, 8999] = float("nan"), float("inf")
    targets = torch.full((M,), 3, dtype=torch.int64, device="cuda")
    r = forward(z, V, 1.0, targets, k)
    dz, _ = backward(z, V, r, 1.0, targets, torch.ones(M, device="cuda"), torch.ones(M, device="cuda"), amax=False)
    torch.cuda.synchronize()
    for row in (0, 2):
        assert torch.isnan(r["logp"][row]) and torch.isnan(r["entropy"][row]) and torch.isnan(r["stats"][row, 1]) and torch.isnan(r["top_logp"][row]).all()
        ids = r["top_ids"][row]
        assert ((ids >= 0) & (ids < V)).all() and len(set(ids.tolist())) == k
        assert torch.isnan(dz[row, :V]).all() and not dz[row, V:].any()
    rest = [i for i in range(M) if i not in (0, 2)]
    assert torch.isfinite(r["logp"][rest]).all() and torch.isfinite(dz[rest].float()).all()
    check_forward(z[1:2], V, {key: v[1:2] for key, v in r.items()}, 1.0, targets[1:2], k)


def test_tokens_that_are_none_or_beyond_the_vocabulary():
    M, V = 4, 1000
    z = make_logits(M, V, 6)
    targets = torch.tensor([-1, V, 5, -100], device="cuda")
    r = forward(z, V, 1.0, targets)
    dz, _ = backward(z, V, r, 1.0, targets, torch.ones(M, device="cuda"), None, amax=False)
    torch.cuda.synchronize()
    assert r["logp"][0].item() == 0 and r["logp"][3].item() == 0 and torch.isnan(r["logp"][1]) and torch.isfinite(r["logp"][2])
    assert not dz[0].any() and not dz[3].any() and torch.isnan(dz[1, :V]).all() and torch.isfinite(dz[2].float()).all()


def test_pitches_in_place_and_no_rows():
    M, V = 11, 1003
    z = make_logits(M, V, 7, pitch=24)
    targets = make_targets(M, V, 7)
    d = torch.randn(M, device="cuda")
    r = forward(z, V, 0.5, targets, 4)
    check_forward(z, V, r, 0.5, targets, 4)
    want, am = backward(z, V, r, 0.5, targets, d, d)
    wider = torch.full((M, 1100 + 4), 9.0, dtype=torch.bfloat16, device="cuda")[:, :1088]
    backward(z, V, r, 0.5, targets, d, d, out=wider)
    torch.cuda.synchronize()
    assert torch.equal(wider[:, :1008], want) and not wider[:, 1008:].any() and (wider.as_strided((M, 16), (1104, 1), 1088) == 9.0).all()
    beside = z.as_strided((M, 24), (1008 + 24, 1), 1008).clone()
    backward(z, V, r, 0.5, targets, d, d, out=z)
    assert torch.equal(z, want)
    assert torch.equal(z.as_strided((M, 24), (1008 + 24, 1), 1008).view(torch.int16), beside.view(torch.int16))
    none = torch.empty((0, 1008), dtype=torch.bfloat16, device="cuda")
    r = forward(none, V, 1.0, torch.empty(0, dtype=torch.int64, device="cuda"), 3)
    _, am = backward(none, V, r, 1.0, torch.empty(0, dtype=torch.int64, device="cuda"), torch.empty(0, device="cuda"), None)
    torch.cuda.synchronize()
    assert am.item() == 0


def test_offsets_beyond_32_bits():
    M, V = 16500, 131072   # 2.16e9 elements
    z = torch.zeros((M, V), dtype=torch.bfloat16, device="cuda")
    z[-3:] = make_logits(3, V, 8)
    z[0] = z[-1]
    targets = torch.full((M,), V - 1, dtype=torch.int64, device="cuda")
    r = forward(z, V, 1.0, targets, 8)
    tail = {k: v[-3:] for k, v in r.items()}
    check_forward(z[-3:], V, tail, 1.0, targets[-3:], 8)
    assert torch.equal(r["top_ids"][0], r["top_ids"][-1]) and r["logp"][0].item() == r["logp"][-1].item()
    small, _ = backward(z[-3:], V, tail, 1.0, targets[-3:], torch.ones(3, device="cuda"), None, amax=False)
    backward(z, V, r, 1.0, targets, torch.ones(M, device="cuda"), None, out=z, amax=False)
    torch.cuda.synchronize()
    assert torch.equal(z[-3:], small) and torch.equal(z[0], small[2])


# ---- distillation ---------------------------------------------------------------------------------

def make_teacher(zw, K, seed, ragged=True):
    """ids the teacher's best on noisy logits, log probabilities of total mass 0.5 .. 0.95; some lists short, some ids twice"""
    g = np.random.default_rng(seed)
    M, V = zw.shape
    ids = np.argsort(-(np.where(zw > -np.inf, zw, -50) + g.normal(size=(M, V))), axis=1)[:, :K].astype(np.int64)
    if ids.shape[1] < K:
        ids = np.concatenate([ids, np.full((M, K - ids.shape[1]), -1)], axis=1)
    t = np.log(g.dirichlet(np.ones(K), size=M) * g.uniform(0.5, 0.95, size=(M, 1)) + 1e-6).astype(np.float32)
    if ragged and M > 3 and K > 3:
        ids[1, 1:] = -1
        ids[2] = -1
        ids[3, 2] = ids[3, 0]
        t[0, 1] = -np.inf
    return np.ascontiguousarray(ids), t


def distill_forward(z, V, ids, t, scale, tail, ts, targets=None, stream=None):
    M = z.shape[0]
    r = dict(stats=torch.full((M, 4), 77.0, device="cuda"), loss=torch.full((M,), 77.0, device="cuda"),
             logp=torch.full((M,), 77.0, device="cuda") if targets is not None else None)
    ws = torch.full((f8.logits_workspace_bytes(M, V),), 255, dtype=torch.uint8, device="cuda")
    f8.distill(z, V, ids, t, r["stats"], r["loss"], targets, r["logp"], tail, ts, scale, ws, stream)
    return r


def distill_backward(z, V, ids, t, r, d_loss, scale, tail, ts, targets=None, d_logp=None, out=None, stream=None):
    dz = out if out is not None else torch.full(z.shape, 9.0, dtype=torch.bfloat16, device="cuda")
    am = torch.full((1,), -1.0, device="cuda")
    f8.distill_bwd(z, V, ids, t, r["stats"], dz, d_loss, targets, d_logp, tail, ts, scale, am, f8.new_workspace(1, 1), stream)
    return dz, am


def check_distill(zw, ids, t, r, dz, am, scale, tail, ts, d_loss, targets, d_logp):
    """Beside the student's errors: the teacher's weights, exp of a value that was scaled and shifted in fp32, are off by a
    factor of 4 u (|t| + 4); the coefficient of the unlisted in the mode with the rest's class, 1 - q_rest / p_rest, by what
    q_rest = 1 - sum q inherits, relative to p_rest."""
    M, V = zw.shape
    dl, fp, p, nl = errors(zw, scale)
    ref = ho.distill(zw, ids, t, scale, tail, ts)
    there = (ids >= 0) & (t > -np.inf)
    tt = np.where(there, t * ts, 0.0)
    q = np.zeros(t.shape)
    for i in range(M):
        cols, w = ho._teacher_row(ids[i], t[i].astype(np.float64), tail, ts)
        q[i, there[i]] = w
    dq = 4 * U * (np.abs(tt).max(axis=1) + 4) + 8 * U               # of every weight, relative
    nlk = np.take_along_axis(nl, np.maximum(ids, 0), axis=1)
    with np.errstate(divide="ignore"):
        lq = np.where(q > 0, np.log(np.where(q > 0, q, 1.0)), 0.0)
    fk = np.take_along_axis(fp, np.maximum(ids, 0), axis=1)
    bound = (q * (2 * dq[:, None] * (1 + np.abs(lq) + nlk) + 2 * fk + 4 * U * nlk)).sum(axis=1) + 2 * dl + 4 * U * np.abs(ref)
    listed = np.zeros((M, V), dtype=bool)
    for i in range(M):
        listed[i, ids[i][ids[i] >= 0]] = True
    dcoef = np.full(M, 4 * U)
    if tail:
        q_rest = np.maximum(1 - q.sum(axis=1), 0)
        p_rest = np.where(listed, 0, p).sum(axis=1)
        f_rest = np.where(listed, 0, p * fp).sum(axis=1) / np.maximum(p_rest, 1e-300) + 2 * dl + (V / 512 + 48) * U
        dr = (q.sum(axis=1) * dq + 4 * U)
        with np.errstate(divide="ignore", invalid="ignore"):
            bound += np.where(q_rest > 0, dr * (1 + np.abs(np.log(q_rest)) + np.abs(np.log(p_rest))) + q_rest * (f_rest + 4 * U * np.abs(np.log(p_rest))) + dr, 0)
            dcoef = np.where(p_rest > 0, (dr + q_rest * (f_rest + 8 * U)) / p_rest + 4 * U, 0.0)
    got, finite = f64(r["loss"]), np.isfinite(ref)   # infinite where a class with weight has no probability
    assert np.array_equal(got[~finite], ref[~finite])
    assert (np.abs(got[finite] - ref[finite]) <= bound[finite]).all(), (np.abs(got[finite] - ref[finite]) / bound[finite]).max()
    rd = ho.distill_bwd(zw, ids, t.astype(np.float64), d_loss, scale, tail, ts, targets, d_logp)
    got = wide(dz)
    assert not got[:, V:].any()
    w = np.abs(d_loss) if d_logp is None else np.abs(d_loss) + np.abs(d_logp) * (targets >= 0)
    qs = np.zeros((M, V))
    for i in range(M):
        np.add.at(qs[i], ids[i][ids[i] >= 0], q[i][ids[i] >= 0])
    with np.errstate(invalid="ignore"):
        coef = np.where(listed, 1.0, np.abs(np.where(p_rest > 0, 1 - q_rest / np.where(p_rest > 0, p_rest, 1), 0.0))[:, None]) if tail else np.ones((M, V))
    bound = HALF * np.abs(rd) + scale * (p * w[:, None] * (1 + coef) * (fp + 16 * U) + np.where(listed, 0, p * (np.abs(d_loss) * dcoef)[:, None])
                                         + np.abs(d_loss)[:, None] * qs * (dq[:, None] + 8 * U))
    bad = np.abs(got[:, :V] - rd) > bound + 1e-38
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])
    assert am.item() == np.abs(got).max(initial=0.0)


@pytest.mark.parametrize("M,V,K", [(1, 100, 1), (5, 37, 37), (6, 513, 128), (40, 5003, 16), (3, 50001, 100), (600, 1000, 8), (4, 131072, 64), (530, 9001, 128),
                                   (4, 140001, 10)])
@pytest.mark.parametrize("tail", (False, True))
def test_distill_against_the_oracle(M, V, K, tail):
    scale, ts = 0.7, 1.0 if tail else 1.4
    z = make_logits(M, V, M * V + K)
    zw = wide(z)[:, :V]
    ids, t = make_teacher(zw, K, V)
    targets = make_targets(M, V, K)
    g = np.random.default_rng(K)
    d_loss, d_logp = (g.normal(size=M).astype(np.float32) for _ in range(2))
    di, dt = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    dv, dw = torch.from_numpy(d_loss).cuda(), torch.from_numpy(d_logp).cuda()
    for hard in (False, True):
        r = distill_forward(z, V, di, dt, scale, tail, ts, targets if hard else None)
        dz, am = distill_backward(z, V, di, dt, r, dv, scale, tail, ts, targets if hard else None, dw if hard else None)
        torch.cuda.synchronize()
        tn = targets.cpu().numpy()
        check_distill(zw, ids, t, r, dz, am, scale, tail, ts, d_loss.astype(np.float64), tn if hard else None, d_logp.astype(np.float64) if hard else None)
        if hard:
            lone = forward(z, V, scale, targets)
            dl, _, _, _ = errors(zw, scale)
            assert (np.abs(f64(r["logp"]) - f64(lone["logp"])) <= 4 * dl + 12 * U * np.abs(f64(lone["logp"]))).all()


@pytest.mark.parametrize("M,V,K", [(6, 1000, 100), (6, 40001, 128), (520, 2001, 128)])
@pytest.mark.parametrize("tail", (False, True))
def test_lists_of_adjacent_and_repeated_tokens(M, V, K, tail):
    """Entries that share their chunk with others: adjacent tokens in any order, across the ends of chunks and pieces of a row; an
    id three times, of which two in one half of the list."""
    g = np.random.default_rng(V)
    z = make_logits(M, V, K)
    zw = wide(z)[:, :V]
    at = np.linspace(0, V - K, M).astype(int)
    ids = np.stack([a + g.permutation(K) for a in at]).astype(np.int64)
    ids[1::2, 5], ids[1::2, K - 1] = ids[1::2, 2], ids[1::2, 2]
    t = np.log(g.dirichlet(np.ones(K), size=M) * 0.8 + 1e-6).astype(np.float32)
    d_loss = g.normal(size=M).astype(np.float32)
    di, dt, dv = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda(), torch.from_numpy(d_loss).cuda()
    r = distill_forward(z, V, di, dt, 0.7, tail, 1.0)
    dz, am = distill_backward(z, V, di, dt, r, dv, 0.7, tail, 1.0)
    torch.cuda.synchronize()
    check_distill(zw, ids, t, r, dz, am, 0.7, tail, 1.0, d_loss.astype(np.float64), None, None)
    for _ in range(5):
        r2 = distill_forward(z, V, di, dt, 0.7, tail, 1.0)
        dz2, am2 = distill_backward(z, V, di, dt, r2, dv, 0.7, tail, 1.0)
        assert torch.equal(r["loss"], r2["loss"]) and torch.equal(r["stats"], r2["stats"]) and torch.equal(dz, dz2) and torch.equal(am, am2)


@pytest.mark.parametrize("M", (4, 560))
def test_distill_masked_students_and_lists(M):
    """A student row with nothing left; listed tokens that the student masks; the whole vocabulary listed; ids beyond it."""
    V, K = 2050, 6
    z = make_logits(M, V, 9)
    z[0] = float("-inf")
    ids = torch.arange(K, device="cuda").repeat(M, 1)
    t = torch.log_softmax(torch.randn(M, K, device="cuda"), dim=1) - 0.1
    z[1, 3] = float("-inf")              # a listed token without probability: an infinite loss, a finite gradient
    z[2, K:V] = float("-inf")            # nothing outside the list
    ids[3, 4] = V
    one = torch.ones(M, device="cuda")
    for tail in (False, True):
        r = distill_forward(z, V, ids, t, 1.0, tail, 1.0)
        dz, _ = distill_backward(z, V, ids, t, r, one, 1.0, tail, 1.0)
        torch.cuda.synchronize()
        loss, d = r["loss"], dz.float()
        assert loss[0].item() == float("inf") and not dz[0].any()
        assert loss[1].item() == float("inf") and torch.isfinite(d[1]).all()
        assert torch.isfinite(d[2]).all() and (loss[2].item() == float("inf")) == tail
        assert torch.isnan(loss[3]) and torch.isnan(d[3, :V]).any()
        if M > 4:
            zw = wide(z[4:])[:, :V]
            check_distill(zw, ids[4:].cpu().numpy(), t[4:].cpu().numpy(), {k: v[4:] if v is not None else None for k, v in r.items()}, dz[4:],
                          dz[4:].float().abs().max().reshape(1), 1.0, tail, 1.0, np.ones(M - 4), None, None)


@pytest.mark.parametrize("M", (5, 560))
@pytest.mark.parametrize("tail", (False, True))
def test_rows_without_entries_have_no_term_whatever_their_logits(M, tail):
    """Masked rows and rows of what memory held, as behind the last sequence; a weight with no row to fall on is no gradient."""
    V, K = 2050, 6
    z = make_logits(M, V, 11)
    z[0], z[1], z[2, 7] = float("-inf"), float("nan"), float("inf")
    ids = torch.full((M, K), -1, dtype=torch.int64, device="cuda")
    t = torch.full((M, K), -2.0, device="cuda")
    if not tail:  # entries that all weigh nothing
        ids[3], t[3] = torch.arange(K, device="cuda"), float("-inf")
    r = distill_forward(z, V, ids, t, 1.0, tail, 1.0)
    dz, am = distill_backward(z, V, ids, t, r, torch.ones(M, device="cuda"), 1.0, tail, 1.0)
    torch.cuda.synchronize()
    assert not r["loss"].any() and not dz.any() and am.item() == 0.0


@pytest.mark.parametrize("M", (5, 560))
@pytest.mark.parametrize("tail", (False, True))
def test_nan_and_infinity_in_a_row_with_entries(M, tail):
    """Also where the teacher gives its entries no weight, so that only the rest's class has a term; other rows stay finite."""
    V, K = 2050, 6
    z = make_logits(M, V, 12)
    z[:, K:V] = z[:, K:V].clamp(-5, 5)
    z[1, 100], z[2, 3] = float("nan"), float("inf")
    ids = torch.arange(K, device="cuda").repeat(M, 1)
    t = torch.full((M, K), -2.5, device="cuda")
    if tail:
        z[3, 200], t[3] = float("inf"), float("-inf")
    r = distill_forward(z, V, ids, t, 1.0, tail, 1.0)
    dz, _ = distill_backward(z, V, ids, t, r, torch.ones(M, device="cuda"), 1.0, tail, 1.0)
    torch.cuda.synchronize()
    bad = [1, 2, 3] if tail else [1, 2]
    fine = [i for i in range(M) if i not in bad]
    assert r["loss"][bad].isnan().all() and dz[bad, :V].isnan().all(dim=1).all()
    masked = torch.isinf(z[fine, :V][:, :K]).any(dim=1)  # (a listed token that the student masks: infinite)
    assert torch.isfinite(r["loss"][fine][~masked]).all() and torch.isfinite(dz[fine].float()).all()


def test_a_teachers_own_pass_feeds_the_student():
    """top_ids and top_logp of one call are the lists of the other; a student that is the teacher has nothing to learn."""
    M, V, K = 12, 4000, 32
    z = make_logits(M, V, 10)
    teacher = forward(z, V, 1.0, None, K, entropy=False)
    r = distill_forward(z, V, teacher["top_ids"], teacher["top_logp"], 1.0, True, 1.0)
    dz, _ = distill_backward(z, V, teacher["top_ids"], teacher["top_logp"], r, torch.ones(M, device="cuda"), 1.0, True, 1.0)
    torch.cuda.synchronize()
    # the loss is second order in the errors of p and q, first order in their sums': some 100 roundings of terms up to log V
    assert r["loss"].abs().max().item() <= 200 * U * np.log(V)
    # q_j - p_j and (1 - q_rest / p_rest) p_j: a few roundings of log p (some 10) in p_j <= 1, and those of the masses
    assert dz.float().abs().max().item() <= 400 * U * 10


@pytest.mark.parametrize("which", ("logprobs", "distill"))
def test_streams_graphs_and_repeats(which):
    M, V, k = 40, 30011, 12
    z = make_logits(M, V, 11)
    targets = make_targets(M, V, 11)
    ids, t = make_teacher(wide(z)[:, :V], k, 11)
    ids, t = torch.from_numpy(ids).cuda(), torch.from_numpy(t).cuda()
    d = torch.randn(M, device="cuda")
    out = dict(stats=torch.empty(M, 2 if which == "logprobs" else 4, device="cuda"), logp=torch.empty(M, device="cuda"), ent=torch.empty(M, device="cuda"),
               loss=torch.empty(M, device="cuda"), ids=torch.empty(M, k, dtype=torch.int64, device="cuda"), top=torch.empty(M, k, device="cuda"),
               dz=torch.empty_like(z), am=torch.empty(1, device="cuda"))
    ws = torch.empty(f8.logits_workspace_bytes(M, V, k), dtype=torch.uint8, device="cuda")

    def step():
        if which == "logprobs":
            f8.token_logprobs(z, V, out["stats"], targets, out["logp"], out["ent"], out["ids"], out["top"], 0.9, ws)
            f8.token_logprobs_bwd(z, V, out["stats"], out["dz"], targets, out["ent"], d, d, 0.9, out["am"], ws)
        else:
            f8.distill(z, V, ids, t, out["stats"], out["loss"], targets, out["logp"], True, 1.0, 0.9, ws)
            f8.distill_bwd(z, V, ids, t, out["stats"], out["dz"], d, targets, d, True, 1.0, 0.9, out["am"], ws)
    written = ["stats", "logp", "dz", "am"] + (["ent", "ids", "top"] if which == "logprobs" else ["loss"])
    snapshot = lambda: {n: out[n].clone().view(torch.uint8) for n in written}
    step()
    torch.cuda.synchronize()
    want = snapshot()
    side = torch.cuda.Stream()
    for n in written:
        out[n].zero_()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
    side.synchronize()
    got = snapshot()
    assert all(torch.equal(got[n], want[n]) for n in written)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        z[:, :V] = (torch.randn(M, V, device="cuda") * (1 + i)).to(torch.bfloat16)
        d.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = snapshot()
        for n in written:
            out[n].zero_()
        step()
        torch.cuda.synchronize()
        want = snapshot()
        assert all(torch.equal(got[n], want[n]) for n in written), i


def test_two_calls_at_once():
    """Streams with workspaces and outputs of their own."""
    V, k = 60000, 20
    z = [make_logits(3, V, 20 + i) for i in range(2)]
    want = [forward(x, V, 1.0, None, k) for x in z]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for x, s in zip(z, streams):
        with torch.cuda.stream(s):
            got.append(forward(x, V, 1.0, None, k))
    torch.cuda.synchronize()
    for a, b in zip(got, want):
        assert all(torch.equal(a[n], b[n]) for n in ("stats", "entropy", "top_ids", "top_logp"))


@pytest.mark.parametrize("V,copies", [(2051, 700), (20003, 600), (60000, 2), (131072, 520)])
def test_equals_beyond_the_room_of_the_selection(V, copies):
    """Rows with more elements at the selection's bound than it has room for, which are then taken from the row's front while the
    block counts them: every wave has to see the same count.  Each copy of a row (a block each, or a row of several blocks) takes
    the same columns, in every pass."""
    k = 128
    at = np.arange(V)
    g = np.random.default_rng(V)
    above = g.permutation(V)
    rows = np.stack([np.zeros(V), np.where(at % 2 == 0, 1.0, -1.0), np.floor(g.random(V) * 3), np.where(at < V - 1500, -np.inf, 2.0),
                     *(np.where(np.isin(at, above[:n]), 4.0 + at % 5, 1.0) for n in (1, 64, 127))])
    n = len(rows)
    z = torch.full((n * copies, (V + 15) // 16 * 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    z[:, :V] = torch.from_numpy(rows.astype(np.float32)).to(torch.bfloat16).cuda().repeat_interleave(copies, dim=0)
    want = torch.from_numpy(np.stack([np.argsort(-wide(z[i * copies:i * copies + 1])[0, :V], kind="stable")[:k] for i in range(n)])).cuda()
    for _ in range(4):
        r = forward(z, V, 1.0, None, k, entropy=False)
        torch.cuda.synchronize()
        assert torch.equal(r["top_ids"], want.repeat_interleave(copies, dim=0))
        assert torch.equal(r["top_logp"], r["top_logp"][::copies].repeat_interleave(copies, dim=0))


@pytest.mark.parametrize("V,copies", [(1000, 60), (9001, 60), (40001, 1), (140001, 1)])
@pytest.mark.parametrize("scale", (1.0, 4.0))
@pytest.mark.parametrize("weight", (1.0, 300.0))
def test_a_rest_far_below_the_list(V, copies, scale, weight):
    """The teacher's remainder has weight where the student puts next to nothing outside the list, or the list lies far below the
    rest: the loss and the gradient are the definition's, however far the two are apart (one exponential of the distance is 0 in
    fp32 from 104 nats on).  Tolerances as above, with the logits outside the list seen from their own largest: every weight there
    is off by a factor of fw, the log of their sum by dl_rest; the distance to the list is taken in fp64 for the loss, and as the
    weights' exponents, off by 4 u of itself, for the gradient."""
    g = np.random.default_rng(V)
    gaps = np.array([0.0, 80.0, 86.9, 87.4, 88.8, 103.5, 105.0, 250.0, 500.0, 1e4, -40.0, -300.0]) / scale
    n, K = len(gaps) + 4, 24
    ids = np.stack([np.sort(g.permutation(V)[:K]) for _ in range(n)]).astype(np.int64)
    listed = np.zeros((n, V), dtype=bool)
    np.put_along_axis(listed, ids, True, axis=1)
    rows = g.normal(size=(n, V)) * 2
    rows[:len(gaps)] -= np.where(listed[:len(gaps)], 0.0, gaps[:, None])
    lowest, part, one, whole = range(len(gaps), n)
    rows[lowest][~listed[lowest]] = LOWEST                                     # all of the rest masked by the lowest value
    rows[part] -= np.where(listed[part], 0.0, 300.0)
    rows[part][~listed[part] & (np.arange(V) % 3 != 0)] = LOWEST               # most of it
    rows[one][~listed[one]] = -np.inf
    rows[one][np.flatnonzero(~listed[one])[V // 2]] = -300.0                   # one left outside the list
    rows[whole] -= np.where(listed[whole], 300.0, np.where(np.arange(V) % 2 == 0, 0.0, 300.0))
    t = np.log(g.dirichlet(np.ones(K), size=n) * g.uniform(0.5, 0.95, size=(n, 1))).astype(np.float32)
    z = torch.full((n, (V + 15) // 16 * 16), float("nan"), dtype=torch.bfloat16)
    z[:, :V] = torch.from_numpy(rows.astype(np.float32)).to(torch.bfloat16)
    zw = wide(z)[:, :V]
    targets = np.where(np.arange(n) % 3 == 0, ids[:, 5], np.where(np.arange(n) % 3 == 1, (ids[:, 0] + 1) % V, -1))
    d_loss, d_logp = (weight * g.normal(size=n)).astype(np.float32), g.normal(size=n).astype(np.float32)
    again = lambda a: torch.from_numpy(np.tile(a, (copies,) + (1,) * (a.ndim - 1))).cuda()
    zc, args = z.repeat(copies, 1).cuda(), [again(a) for a in (ids, t)]
    tg, dv, dw = again(targets), again(d_loss), again(d_logp)
    r = distill_forward(zc, V, *args, scale, True, 1.0, tg)
    dz, am = distill_backward(zc, V, *args, r, dv, scale, True, 1.0, tg, dw)
    torch.cuda.synchronize()
    for v in (*r.values(), dz):  # every copy alike
        assert torch.equal(v, v[:n].repeat((copies,) + (1,) * (v.dim() - 1)))

    dl, fp, p, nl = errors(zw, scale)
    ref = ho.distill(zw, ids, t.astype(np.float64), scale, True)
    q = np.exp(t.astype(np.float64))
    q_rest = 1 - q.sum(axis=1)
    dq = 4 * U * (np.abs(t).max(axis=1) + 4) + 8 * U
    dr = q.sum(axis=1) * dq + 4 * U
    rest = np.where(listed, -np.inf, zw)
    dl_rest, fw, w, nl_rest = errors(rest, scale)
    logs = nl.min(axis=1) + nl_rest.min(axis=1) + np.abs(np.log(q_rest))      # magnitudes of the logs of sums and masses, together
    apart = scale * np.abs(zw.max(axis=1) - rest.max(axis=1))
    nlk, fk = np.take_along_axis(nl, ids, axis=1), np.take_along_axis(fp, ids, axis=1)
    fk = np.maximum(fk, 4 * U * nlk)    # (errors() ends its exponents at 800)
    bound = ((q * (2 * dq[:, None] * (1 + np.abs(t) + nlk) + 2 * fk + 4 * U * nlk)).sum(axis=1) + 2 * dl + 2 * dl_rest + dr * (2 + logs + apart)
             + q_rest * 8 * U * (1 + logs) + 4 * U * np.abs(ref))
    got = f64(r["loss"][:n])
    with np.errstate(over="ignore"):
        dead = ref.astype(np.float32) == np.inf   # (the lowest value, scaled)
    assert np.array_equal(got == np.inf, dead)
    assert (np.abs(got - ref) <= bound)[~dead].all(), (got, ref, bound)

    rd = ho.distill_bwd(zw, ids, t.astype(np.float64), d_loss.astype(np.float64), scale, True, 1.0, targets, d_logp.astype(np.float64))
    got = wide(dz[:n])
    assert np.isfinite(got).all() and not got[:, V:].any()
    gl, gt = np.abs(d_loss.astype(np.float64))[:, None], (np.abs(d_logp.astype(np.float64)) * (targets >= 0))[:, None]
    qs = np.zeros((n, V))
    np.put_along_axis(qs, ids, q, axis=1)
    # p outside the list is its weight there times r = p_rest / q_rest, an exponential of a sum of four terms
    fr = (4 * U * np.minimum(apart, 800) + dl + dl_rest + 8 * U * (1 + logs) + dr / q_rest)[:, None]
    bound = HALF * np.abs(rd) + scale * np.where(listed, p * (gl + gt) * (fp + 16 * U) + gl * qs * (dq[:, None] + 8 * U),
                                                 gl * w * q_rest[:, None] * (fw + (dr / q_rest + 8 * U * (1 + logs))[:, None]) + p * (gl + gt) * (fp + fw + fr + 16 * U))
    bad = np.abs(got[:, :V] - rd) > bound + 1e-37 * (1 + weight)
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4])
    assert am.item() == np.abs(got).max()


# ---- the kernels of large tensors -------------------------------------------------------------------

def large_logits(M, V, seed):
    torch.manual_seed(seed)
    z = torch.full((M, (V + 15) // 16 * 16), float("nan"), dtype=torch.bfloat16, device="cuda")
    for rows in z.split(1024):
        rows[:, :V] = torch.randn((len(rows), V), device="cuda") * 3
    return z


def parts_of(M, n=300):
    """Calls of n rows, whose rows are cut for the forward as those of all and which load through the caches."""
    return [slice(i, i + n) for i in range(0, M - n, n)] + [slice(M - n, M)]


# The forward loads past the caches from 2^29 elements on; the gradient from 2^27 on, in blocks of 1024 threads where there are 2048 rows
# or pieces of rows as long as those blocks' steps: with both, of many long rows; one of the two alone in the last two cases.
@pytest.mark.parametrize("M,V", [(4200, 131071), (2700, 50001), (2100, 32768), (600, 262144)])
@pytest.mark.parametrize("entropy", (False, True))
def test_large_logits_have_the_bits_of_their_rows(M, V, entropy):
    z = large_logits(M, V, 31)
    targets = torch.randint(-1, V, (M,), device="cuda")
    d_logp, d_entropy = torch.randn(M, device="cuda"), torch.randn(M, device="cuda") if entropy else None
    r = forward(z, V, 0.8, targets, 0, entropy)
    dz, am = backward(z, V, r, 0.8, targets, d_logp, d_entropy)
    torch.cuda.synchronize()
    for rows in parts_of(M):
        at = lambda t: None if t is None else t[rows]
        pr = forward(z[rows], V, 0.8, targets[rows], 0, entropy)
        pz, _ = backward(z[rows], V, pr, 0.8, targets[rows], d_logp[rows], at(d_entropy))
        torch.cuda.synchronize()
        assert torch.equal(pz, dz[rows]) and all(v is None or torch.equal(v, r[k][rows]) for k, v in pr.items())
    assert am.item() == max(t.float().abs().max().item() for t in dz.split(1024))
    few = {k: v[:3] if v is not None else None for k, v in r.items()}
    check_forward(z[:3], V, few, 0.8, targets[:3], 0)
    zw, t = wide(z[:3])[:, :V], targets[:3].cpu().numpy()
    wl, wh = np.abs(f64(d_logp[:3])) * (t >= 0), f64(d_entropy[:3]) if entropy else None
    check_gradient(zw, V, dz[:3], None, ho.token_logprobs_bwd(zw, 0.8, t, f64(d_logp[:3]), wh), 0.8, wl, np.abs(wh) if entropy else None)
    backward(z, V, r, 0.8, targets, d_logp, d_entropy, out=z)   # in place
    torch.cuda.synchronize()
    assert torch.equal(z, dz)


# With a teacher blocks of 1024 threads take rows of 98304 columns and more.
@pytest.mark.parametrize("M,V,K", [(4200, 131071, 64), (2100, 98304, 128), (2700, 50001, 100)])
@pytest.mark.parametrize("tail", (False, True))
def test_distill_of_large_logits_has_the_bits_of_its_rows(M, V, K, tail):
    scale, ts = 0.7, 1.0 if tail else 1.4
    z = large_logits(M, V, 32)
    ids = torch.randint(0, V, (M, K), device="cuda")
    ids[:, K // 2:] = torch.sort(torch.rand((M, V // 64), device="cuda"), dim=1).indices[:, :K - K // 2] + 17   # some close together
    ids[::5, K - 3:], ids[1::5, 4] = -1, ids[1::5, 1]
    t = torch.log_softmax(torch.randn((M, K), device="cuda"), dim=1) - 0.3
    targets = torch.randint(-1, V, (M,), device="cuda")
    d_loss, d_logp = torch.randn(M, device="cuda"), torch.randn(M, device="cuda")
    r = distill_forward(z, V, ids, t, scale, tail, ts, targets)
    dz, am = distill_backward(z, V, ids, t, r, d_loss, scale, tail, ts, targets, d_logp)
    torch.cuda.synchronize()
    for rows in parts_of(M):
        pr = distill_forward(z[rows], V, ids[rows], t[rows], scale, tail, ts, targets[rows])
        pz, _ = distill_backward(z[rows], V, ids[rows], t[rows], pr, d_loss[rows], scale, tail, ts, targets[rows], d_logp[rows])
        torch.cuda.synchronize()
        assert torch.equal(pz, dz[rows]) and all(torch.equal(v, r[k][rows]) for k, v in pr.items())
    assert am.item() == max(x.float().abs().max().item() for x in dz.split(1024))
    n = 6
    check_distill(wide(z[:n])[:, :V], ids[:n].cpu().numpy(), t[:n].cpu().numpy(), {k: v[:n] for k, v in r.items()}, dz[:n],
                  dz[:n].float().abs().max().reshape(1), scale, tail, ts, f64(d_loss[:n]), targets[:n].cpu().numpy(), f64(d_logp[:n]))
    distill_backward(z, V, ids, t, r, d_loss, scale, tail, ts, targets, d_logp, out=z)   # in place
    torch.cuda.synchronize()
    assert torch.equal(z, dz)
