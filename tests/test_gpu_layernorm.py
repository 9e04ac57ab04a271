"""f8.layernorm and its backward through the C ABI against oracle/step_oracle.py (fp64).

Tolerances.  A result in bf16 is off by half a step, 2^-8 of its value, plus what fp32 arithmetic leaves.  A sum over a row of
D <= 16384 terms takes at most 16 + 6 + 16 additions one after the other (a thread's terms, lanes, waves), so it is off by less
than 2^-18 of the sum of magnitudes; FP is 2^-17 of the magnitudes that enter, in each place where terms can cancel.  A row's
differences from its mean carry 2^-18 of its mean magnitude A, so with the deviation 1 / rstd the statistics are off by
FP (1 + rstd A) relative.  Sums over rows: one addition per row of a block, then per block and group, 2^-24 of the sum of
magnitudes each."""
import numpy as np
import pytest
import torch

import oracle as o
from oracle import step_oracle as so
from paper_2410_06511_amd import f8
from helpers import bits

pytestmark = pytest.mark.gpu

EPS = 1e-5
HALF, FP = 2.0 ** -8, 2.0 ** -17


def gen(shape, seed, std=1.0, mean=0.0):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std + mean).to(torch.bfloat16)


def wide(t):
    return None if t is None else o.bf16_to_f32(bits(t)).astype(np.float64) if t.dtype == torch.bfloat16 else t.cpu().numpy().astype(np.float64)


def rows(M, D, seed=None, std=1.0, mean=0.0, pitch=0):
    t = torch.full((M, D + pitch), 7.0, dtype=torch.bfloat16, device="cuda")
    if seed is not None:
        t[:, :D] = gen((M, D), seed, std, mean).cuda()
    return t[:, :D]


def make(M, D, residual, bias, seed=0, pitch=0, mean=0.4):
    return dict(x=rows(M, D, seed * 100 + 1, 1.0, mean, pitch), y=rows(M, D, seed * 100 + 2, 0.5, 0.0, pitch) if residual else None,
                g=gen((D,), seed + 3, 0.2, 1.0).cuda(), b=gen((D,), seed + 4, 0.3).cuda() if bias else None,
                dn=rows(M, D, seed * 100 + 5, 1e-2, 0.0, pitch), dh=rows(M, D, seed * 100 + 6, 1e-2, 0.0, pitch))


def forward(s, M, D, pitch=0, stream=None, amax=True):
    f32 = lambda n: torch.full((n,), 5.0, device="cuda")
    r = dict(h=rows(M, D, pitch=pitch) if s["y"] is not None else None, n=rows(M, D, pitch=pitch), mean=f32(M), rstd=f32(M), amax=f32(1) if amax else None)
    ws = f8.new_workspace(max(M, 1), D)
    if stream is not None:
        torch.cuda.synchronize()   # what was filled above was filled on the current stream
    f8.layernorm(s["x"], s["g"], r["n"], s["b"], s["y"], r["h"], EPS, r["mean"], r["rstd"], r["amax"], ws, stream)
    if stream is not None:
        torch.cuda.synchronize()
    return r


def backward(s, r, M, D, add=True, pitch=0, stream=None):
    f32 = lambda n: torch.full((n,), 5.0, device="cuda")
    g = dict(dx=rows(M, D, pitch=pitch), dg=f32(D), db=f32(D), amax=f32(1))
    ws = torch.full((f8.layernorm_bwd_workspace_bytes(M, D),), 255, dtype=torch.uint8, device="cuda")
    if stream is not None:
        torch.cuda.synchronize()
    f8.layernorm_bwd(s["x"] if r["h"] is None else r["h"], s["g"], r["mean"], r["rstd"], s["dn"], g["dx"], s["dh"] if add else None, g["dg"], g["db"], g["amax"],
                     ws, stream)
    if stream is not None:
        torch.cuda.synchronize()
    return g


def kept(s, r):
    return wide(s["x"] if r["h"] is None else r["h"])


def check_forward(s, r):
    if s["y"] is not None:
        assert torch.equal(r["h"], (s["x"].float() + s["y"].float()).to(torch.bfloat16))
    h, g, b = kept(s, r), wide(s["g"]), wide(s["b"])
    n, mean, rstd = so.layernorm(h, g, b, EPS)
    a = np.abs(h).mean(axis=1)
    assert (np.abs(wide(r["mean"]) - mean) <= FP * a).all()
    rel = FP * (1 + rstd * a)
    assert (np.abs(wide(r["rstd"]) - rstd) <= rel * rstd).all()
    part = n if b is None else n - b
    bound = HALF * np.abs(n) + 2 * rel[:, None] * np.abs(part) + FP * (np.abs(g) * (rstd * a)[:, None] + np.abs(g * h) * rstd[:, None])
    assert (np.abs(wide(r["n"]) - n) <= (bound if b is None else bound + FP * np.abs(b))).all()
    if r["amax"] is not None:
        assert r["amax"].item() == (np.abs(wide(r["n"])).max() if h.size else 0.0)


def check_backward(s, r, g, add=True):
    h, gain, dn, dh = kept(s, r), wide(s["g"]), wide(s["dn"]), wide(s["dh"]) if add else None
    M, D = h.shape
    dx, dg, db = so.layernorm_bwd(h, gain, dn, dh, EPS)
    _, mean, rstd = so.layernorm(h, gain, None, EPS)
    a = np.abs(h).mean(axis=1, keepdims=True)
    rstd = rstd[:, None]
    slack = FP * (1 + rstd * a)
    c, w = rstd * (np.abs(h) + a), np.abs(gain * dn)
    md = rstd * (w + w.mean(axis=1, keepdims=True) + c * (w * c).mean(axis=1, keepdims=True))
    assert (np.abs(wide(g["dx"]) - dx) <= HALF * np.abs(dx) + 4 * slack * md + (0 if dh is None else FP * np.abs(dh)) + 1e-38).all()
    adds = 2.0 ** -24 * (M / 256 + 66)
    assert (np.abs(wide(g["dg"]) - dg) <= ((adds + 2 * slack) * np.abs(dn) * c).sum(axis=0) + 1e-38).all()
    assert (np.abs(wide(g["db"]) - db) <= adds * np.abs(dn).sum(axis=0) + 1e-38).all()
    assert g["amax"].item() == (np.abs(wide(g["dx"])).max() if h.size else 0.0)


# one row, rows beyond a block's, every shape of a row (a wave's with one and two chunks, blocks of each size), odd sizes
SIZES = [(0, 64), (1, 8), (3, 72), (5, 512), (9, 520), (1000, 1024), (4, 1032), (7, 2816), (2500, 2056), (3, 4096), (5, 4104), (2, 8192), (3, 8200), (2, 12288), (2, 16384)]


@pytest.mark.parametrize("M,D", SIZES)
@pytest.mark.parametrize("residual,bias", [(False, False), (False, True), (True, True)])
def test_against_the_oracle(M, D, residual, bias):
    s = make(M, D, residual, bias, seed=M % 7 + D % 5)
    r = forward(s, M, D)
    check_forward(s, r)
    for add in (True, False):
        check_backward(s, r, backward(s, r, M, D, add), add)


@pytest.mark.parametrize("M,D", [(9, 264), (6, 2816), (3, 8200)])
def test_row_pitches(M, D):
    s = make(M, D, True, True, pitch=24)
    r = forward(s, M, D, pitch=40)
    g = backward(s, r, M, D, pitch=8)
    check_forward(s, r), check_backward(s, r, g)
    for t in (r["h"], r["n"], g["dx"]):    # what lies between the rows is left alone
        full = t.as_strided((M, t.stride(0)), (t.stride(0), 1))
        assert bool((full[:M - 1, D:] == 7.0).all())


def test_large_tensors():
    """Loads past the caches; more rows than blocks."""
    M, D = 16400, 2056
    s = make(M, D, False, True)
    r = forward(s, M, D)
    check_forward(s, r), check_backward(s, r, backward(s, r, M, D))


def test_a_mean_far_from_zero():
    M, D = 6, 1024
    s = make(M, D, False, True, mean=200.0)
    r = forward(s, M, D)
    check_forward(s, r), check_backward(s, r, backward(s, r, M, D))


def test_constant_rows_and_rows_that_are_not_numbers():
    M, D = 6, 512
    s = make(M, D, False, True)
    s["x"][1] = 3.0
    s["x"][3, 17] = float("nan")
    s["x"][4, 5] = float("inf")
    r = forward(s, M, D, amax=False)
    assert torch.equal(r["n"][1], s["b"]) and r["mean"][1].item() == 3.0
    assert abs(r["rstd"][1].item() - EPS ** -0.5) < 1e-4 * EPS ** -0.5
    assert bool(r["n"][3].isnan().all()) and bool(r["n"][4].isnan().any()) and bool(r["n"][[0, 1, 2, 5]].isfinite().all())


def test_outputs_in_the_place_of_inputs():
    M, D = 37, 2816
    for residual in (False, True):
        s = make(M, D, residual, True)
        r = forward(s, M, D)
        g = backward(s, r, M, D)
        t = {k: None if v is None else v.clone() for k, v in s.items()}
        mean, rstd = torch.empty(M, device="cuda"), torch.empty(M, device="cuda")
        if residual:
            f8.layernorm(t["x"], t["g"], t["y"], t["b"], t["y"], t["x"], EPS, mean, rstd)   # h over x, n over y
            assert torch.equal(t["x"], r["h"]) and torch.equal(t["y"], r["n"])
        else:
            f8.layernorm(t["x"], t["g"], t["x"], t["b"], None, None, EPS, mean, rstd)
            assert torch.equal(t["x"], r["n"])
        for into in ("dn", "dh", "h"):
            u = dict(dn=s["dn"].clone(), dh=s["dh"].clone(), h=(s["x"] if r["h"] is None else r["h"]).clone())
            f8.layernorm_bwd(u["h"], s["g"], r["mean"], r["rstd"], u["dn"], u[into], u["dh"])
            assert torch.equal(u[into], g["dx"])


def test_single_outputs():
    M, D = 50, 768
    s = make(M, D, False, True)
    r = forward(s, M, D)
    g = backward(s, r, M, D, add=False)
    n = rows(M, D)
    f8.layernorm(s["x"], s["g"], n, s["b"])
    assert torch.equal(n, r["n"])
    ws = torch.empty(f8.layernorm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    dx, dg, db = rows(M, D), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    f8.layernorm_bwd(s["x"], s["g"], r["mean"], r["rstd"], s["dn"], dx)
    f8.layernorm_bwd(s["x"], s["g"], r["mean"], r["rstd"], s["dn"], dg=dg, workspace=ws)
    f8.layernorm_bwd(s["x"], s["g"], r["mean"], r["rstd"], s["dn"], db=db, workspace=ws)
    assert torch.equal(dx, g["dx"]) and torch.equal(dg, g["dg"]) and torch.equal(db, g["db"])


def test_on_another_stream_and_in_a_graph():
    M, D = 300, 1536
    batches = [make(M, D, True, True, seed=i) for i in range(3)]
    eager = [(forward(s, M, D), None) for s in batches]
    eager = [(r, backward(s, r, M, D)) for s, (r, _) in zip(batches, eager)]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    r = forward(batches[0], M, D, stream=side)
    g = backward(batches[0], r, M, D, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(r["n"], eager[0][0]["n"]) and torch.equal(g["dg"], eager[0][1]["dg"])
    s = {k: v.clone() for k, v in batches[0].items()}
    out = dict(h=rows(M, D), n=rows(M, D), mean=torch.empty(M, device="cuda"), rstd=torch.empty(M, device="cuda"), amax=torch.empty(1, device="cuda"))
    grad = dict(dx=rows(M, D), dg=torch.empty(D, device="cuda"), db=torch.empty(D, device="cuda"), amax=torch.empty(1, device="cuda"))
    ws = torch.empty(f8.layernorm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        f8.layernorm(s["x"], s["g"], out["n"], s["b"], s["y"], out["h"], EPS, out["mean"], out["rstd"], out["amax"], ws)
        f8.layernorm_bwd(out["h"], s["g"], out["mean"], out["rstd"], s["dn"], grad["dx"], s["dh"], grad["dg"], grad["db"], grad["amax"], ws)
    for i in (0, 1, 2, 1):
        for k, v in s.items():
            v.copy_(batches[i][k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.randn(1 << 20, device="cuda").sum().isfinite().item()
        for k in ("h", "n", "mean", "rstd", "amax"):
            assert torch.equal(out[k], eager[i][0][k]), k
        for k in ("dx", "dg", "db", "amax"):
            assert torch.equal(grad[k], eager[i][1][k]), k


def test_gradients_by_differences():
    """Of a smooth loss through the kernels' own forward: outputs in bf16 limit it to some per cent."""
    M, D = 4, 256
    s = make(M, D, False, True, mean=0.0)
    r = forward(s, M, D)
    g = backward(s, r, M, D, add=False)
    direction = torch.randn((M, D), generator=torch.Generator().manual_seed(9)).to(torch.bfloat16).cuda()
    step = 0.25
    loss = []
    for sign in (1, -1):
        x = (s["x"].double() + sign * step * direction.double()).to(torch.bfloat16)
        n = rows(M, D)
        f8.layernorm(x, s["g"], n, s["b"])
        loss.append((n.double() * s["dn"].double()).sum().item())
    moved = ((s["x"].double() + step * direction.double()).to(torch.bfloat16).double() - (s["x"].double() - step * direction.double()).to(torch.bfloat16).double())
    want = (g["dx"].double() * moved).sum().item()
    # rounding of n: 2^-8 of each of the products' terms, independent; third derivatives: (step)^2 / 6 of the terms' size
    noise = 2 * HALF * ((s["dn"].double() * r["n"].double()).square().sum().sqrt().item()) * 4 + step ** 2 * (g["dx"].double() * moved).norm().item()
    assert abs(loss[0] - loss[1] - want) <= noise
