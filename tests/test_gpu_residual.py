"""f8.residual_norm and its backward through the C ABI against oracle/head_oracle.py (fp64).

Tolerances.  A result in bf16 is off by half a step, 2^-8 of its value, plus what fp32 arithmetic leaves: a sum over a row of D
terms takes at most D / 512 + 14 additions one after the other (chunks of 8, then lanes by halves) of 2^-24 each, at most 2^-18
for D <= 16384; a handful of products add less.  FP is 2^-17 of the magnitudes that enter, in each place where terms can cancel.
Sums over rows: one addition per row of a block, then per block and group, 2^-24 of the sum of magnitudes each."""
import numpy as np
import pytest
import torch

import oracle as o
from oracle import head_oracle as ho
from paper_2410_06511_amd import f8
from paper_2410_06511_amd import workloads as wl
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


def make(M, D, post, gates, pre, seed=0, pitch=0):
    """Inputs on the GPU; pitch: extra columns of every matrix."""
    def rows(salt, std):
        t = torch.full((M, D + pitch), 7.0, dtype=torch.bfloat16, device="cuda")
        t[:, :D] = gen((M, D), seed * 100 + salt, std).cuda()
        return t[:, :D]
    return dict(x=rows(1, 1.0), y=rows(2, 0.5), dh=rows(3, 1e-2), dn=rows(4, 1e-2) if pre else None,
                g_post=gen((D,), seed + 5, 0.2, 1.0).cuda() if post else None, gate=gen((gates, D), seed + 6, 0.5, 0.5).cuda() if gates else None,
                g_pre=gen((D,), seed + 7, 0.2, 1.0).cuda() if pre else None)


def out_rows(M, D, pitch=0):
    return torch.full((M, D + pitch), -3.0, dtype=torch.bfloat16, device="cuda")[:, :D]


def run_forward(s, M, D, a, b, amax=True, pitch=0, stream=None):
    r = dict(h=out_rows(M, D, pitch), n=out_rows(M, D, pitch) if s["g_pre"] is not None else None)
    f32 = lambda *sh: torch.empty(sh, device="cuda")
    r["rstd_post"] = f32(M) if s["g_post"] is not None else None
    r["rstd_pre"] = f32(M) if s["g_pre"] is not None else None
    r["amax_n"] = f32(1) if amax and s["g_pre"] is not None else None
    f8.residual_norm(s["x"], s["y"], r["h"], r["n"], s["g_post"], s["gate"], s["g_pre"], a, b, EPS, r["rstd_post"], r["rstd_pre"], r["amax_n"],
                     f8.new_workspace(max(M, 1), D), stream)
    return r


def run_backward(s, r, M, D, a, b, pitch=0, no_dh=False, stream=None):
    gates = 0 if s["gate"] is None else s["gate"].shape[0]
    f32 = lambda *sh: torch.full(sh, 5.0, device="cuda")
    g = dict(dx=out_rows(M, D, pitch), dy=out_rows(M, D, pitch), dg_post=f32(D) if s["g_post"] is not None else None,
             dgate=f32(gates, D) if gates else None, dg_pre=f32(D) if s["g_pre"] is not None else None, amax_dy=f32(1))
    ws = torch.full((f8.residual_norm_bwd_workspace_bytes(M, D, gates),), 255, dtype=torch.uint8, device="cuda")
    f8.residual_norm_bwd(s["y"], g["dx"], g["dy"], h=r["h"], dh=None if no_dh else s["dh"], dn=s["dn"], g_post=s["g_post"], gate=s["gate"],
                         g_pre=s["g_pre"], skip_scale=a, branch_scale=b, rstd_post=r["rstd_post"], rstd_pre=r["rstd_pre"], dg_post=g["dg_post"],
                         dgate=g["dgate"], dg_pre=g["dg_pre"], amax_dy=g["amax_dy"], workspace=ws, stream=stream)
    return g


def check_forward(s, r, a, b):
    x, y, g_post, gate, g_pre = (wide(s[k]) for k in ("x", "y", "g_post", "gate", "g_pre"))
    M, D = x.shape
    h, r1 = ho.residual_h(x, y, g_post, gate, a, b, EPS)
    branch, _ = ho.residual_h(0 * x, y, g_post, gate, a, b, EPS)
    got = wide(r["h"])
    assert (np.abs(got - h) <= HALF * np.abs(h) + FP * (np.abs(a * x) + np.abs(branch))).all()
    if r1 is not None:
        assert np.allclose(wide(r["rstd_post"]), r1, rtol=2.0 ** -18, atol=0)
    if g_pre is not None:
        n, r2 = ho.norm(got, g_pre, EPS)
        assert np.allclose(wide(r["rstd_pre"]), r2, rtol=2.0 ** -18, atol=0)
        assert (np.abs(wide(r["n"]) - n) <= (HALF + FP) * np.abs(n)).all()
        if r["amax_n"] is not None:
            assert r["amax_n"].item() == (np.abs(wide(r["n"])).max() if M else 0.0)


def check_backward(s, r, g, a, b, no_dh=False):
    y, g_post, gate, g_pre, dh, dn, h = (wide(v) for v in (s["y"], s["g_post"], s["gate"], s["g_pre"], s["dh"], s["dn"], r["h"]))
    M, D = y.shape
    if no_dh:
        dh = None
    ref = ho.residual_bwd(h, y, dh, dn, g_post, gate, g_pre, a, b, EPS)
    # magnitudes of the terms of t, of the branch's gradient v, and of dy
    mt = np.zeros((M, D)) if dh is None else np.abs(dh)
    if g_pre is not None:
        r2 = wide(r["rstd_pre"])[:, None]
        w = np.abs(dn * g_pre)
        mt = mt + r2 * w + np.abs(h) * r2 ** 3 * (np.abs(h) * w).mean(axis=1, keepdims=True)
    assert (np.abs(wide(g["dx"]) - ref["dx"]) <= HALF * np.abs(ref["dx"]) + FP * abs(a) * mt + 1e-38).all()
    gr = ho._gate_rows(gate, M, D)
    mv = np.abs(b * gr) * mt
    u = y if g_post is None else y * wide(r["rstd_post"])[:, None] * g_post
    md = mv
    if g_post is not None:
        r1 = wide(r["rstd_post"])[:, None]
        w = mv * np.abs(g_post)
        md = r1 * w + np.abs(y) * r1 ** 3 * (np.abs(y) * w).mean(axis=1, keepdims=True)
    assert (np.abs(wide(g["dy"]) - ref["dy"]) <= HALF * np.abs(ref["dy"]) + 2 * FP * md + 1e-38).all()
    assert g["amax_dy"].item() == (np.abs(wide(g["dy"])).max() if M else 0.0)
    adds = 2.0 ** -24 * (M / 512 + 64 + 2) + 2 * FP
    if g_pre is not None:
        assert (np.abs(wide(g["dg_pre"]) - ref["dg_pre"]) <= adds * np.abs(dn * h * wide(r["rstd_pre"])[:, None]).sum(axis=0) + 1e-38).all()
    if g_post is not None:
        assert (np.abs(wide(g["dg_post"]) - ref["dg_post"]) <= adds * (mv * np.abs(y) * wide(r["rstd_post"])[:, None]).sum(axis=0) + 1e-38).all()
    if gate is not None:
        G = gate.shape[0]
        rows = M // G
        adds = 2.0 ** -24 * (rows + 66) + 2 * FP   # (a block may take a whole group)
        assert (np.abs(wide(g["dgate"]) - ref["dgate"]) <= adds * (np.abs(b) * mt * np.abs(u)).reshape(G, -1, D).sum(axis=1) + 1e-38).all()


# every width class of the kernels, odd sizes, one token to many; gates: none, per channel, per sequence, per token
CASES = [(1, 8, True, 0, True), (1, 4096, True, 1, True), (3, 40, False, 0, True), (7, 512, True, 7, True), (65, 520, True, 5, True),
         (130, 1024, False, 1, True), (33, 1032, True, 0, False), (600, 2048, True, 3, True), (515, 2816, False, 0, False), (40, 4096, True, 40, True),
         (12, 4104, True, 1, True), (100, 8192, True, 4, True), (9, 8200, True, 1, True), (5, 16384, True, 5, True), (6, 16384, False, 1, False),
         (1100, 256, True, 1100, True), (2600, 64, True, 2, True)]


@pytest.mark.parametrize("M,D,post,gates,pre", CASES)
def test_against_the_oracle(M, D, post, gates, pre):
    a, b = 0.75, 1.5
    s = make(M, D, post, gates, pre, M + D)
    r = run_forward(s, M, D, a, b)
    g = run_backward(s, r, M, D, a, b)
    torch.cuda.synchronize()
    check_forward(s, r, a, b)
    check_backward(s, r, g, a, b)


def test_row_pitches_and_what_lies_between_rows():
    M, D = 37, 136
    s = make(M, D, True, 1, True, 3, pitch=24)
    r = run_forward(s, M, D, 1.0, 1.0, pitch=8)
    g = run_backward(s, r, M, D, 1.0, 1.0, pitch=40)
    torch.cuda.synchronize()
    check_forward(s, r, 1.0, 1.0)
    check_backward(s, r, g, 1.0, 1.0)
    for t, extra in ((r["h"], 8), (r["n"], 8), (g["dx"], 40), (g["dy"], 40)):
        assert (t.as_strided((M, extra), (D + extra, 1), D) == -3.0).all()


def test_gradient_of_the_norm_alone():
    """No gradient of h itself (the last block's norm in front of the output projection)."""
    M, D = 50, 768
    s = make(M, D, False, 0, True, 4)
    r = run_forward(s, M, D, 1.0, 1.0)
    g = run_backward(s, r, M, D, 1.0, 1.0, no_dh=True)
    torch.cuda.synchronize()
    check_backward(s, r, g, 1.0, 1.0, no_dh=True)
    assert torch.equal(g["dx"], g["dy"])


@pytest.mark.parametrize("M,D", [(16, 16), (272, 336), (1008, 1024), (48, 4096), (64, 8192), (32, 12288), (16, 16384)])
def test_plain_residual_and_norm_have_the_bits_of_add_and_rmsnorm(M, D):
    s = make(M, D, False, 0, True, 5)
    r = run_forward(s, M, D, 1.0, 1.0)
    h, n, rstd, amax = torch.empty_like(s["x"]), torch.empty_like(s["x"]), torch.empty(M, device="cuda"), torch.empty(1, device="cuda")
    f8.add(s["x"], s["y"], h)
    f8.rmsnorm(h, s["g_pre"], EPS, n, rstd, amax, f8.new_workspace(M, D))
    torch.cuda.synchronize()
    assert torch.equal(r["h"].view(torch.int16), h.view(torch.int16)) and torch.equal(r["n"].view(torch.int16), n.view(torch.int16))
    assert torch.equal(r["rstd_pre"], rstd) and torch.equal(r["amax_n"], amax)


def test_in_place():
    M, D, a, b = 66, 640, 1.0, 0.5
    s = make(M, D, True, 2, True, 6)
    want = run_forward(s, M, D, a, b)
    grads = run_backward(s, want, M, D, a, b)
    torch.cuda.synchronize()
    x, y = s["x"].clone(), s["y"].clone()
    f8.residual_norm(x, y, x, y, s["g_post"], s["gate"], s["g_pre"], a, b, EPS)   # h over x, n over y
    assert torch.equal(x, want["h"]) and torch.equal(y, want["n"])
    y = s["y"].clone()
    f8.residual_norm(s["x"], y, y, torch.empty_like(y), s["g_post"], s["gate"], s["g_pre"], a, b, EPS)  # h over y
    assert torch.equal(y, want["h"])
    for over in ("dn", "y", "h"):
        dh, t = s["dh"].clone(), {"dn": s["dn"].clone(), "y": s["y"].clone(), "h": want["h"].clone()}
        f8.residual_norm_bwd(t["y"], dh, t[over], h=t["h"], dh=dh, dn=t["dn"], g_post=s["g_post"], gate=s["gate"], g_pre=s["g_pre"], skip_scale=a,
                             branch_scale=b, rstd_post=want["rstd_post"], rstd_pre=want["rstd_pre"])
        assert torch.equal(dh, grads["dx"]) and torch.equal(t[over], grads["dy"]), over


def test_single_outputs_have_the_bits_of_all_together():
    M, D = 70, 1536
    s = make(M, D, True, 1, True, 8)
    r = run_forward(s, M, D, 1.0, 1.0)
    g = run_backward(s, r, M, D, 1.0, 1.0)
    kw = dict(h=r["h"], dh=s["dh"], dn=s["dn"], g_post=s["g_post"], gate=s["gate"], g_pre=s["g_pre"], rstd_post=r["rstd_post"], rstd_pre=r["rstd_pre"])
    ws = torch.empty(f8.residual_norm_bwd_workspace_bytes(M, D, 1), dtype=torch.uint8, device="cuda")
    for name in ("dx", "dy", "dg_post", "dgate", "dg_pre"):
        t = torch.zeros_like(g[name])
        outs = {k: (t if k == name else None) for k in ("dx", "dy", "dg_post", "dgate", "dg_pre")}
        f8.residual_norm_bwd(s["y"], outs.pop("dx"), outs.pop("dy"), workspace=ws, **outs, **kw)
        assert torch.equal(t, g[name]), name
    # and again: the same bits
    again = run_backward(s, r, M, D, 1.0, 1.0)
    assert all(torch.equal(again[k], g[k]) for k in g)


def test_no_rows():
    D = 64
    s = make(0, D, True, 2, True, 9)
    r = run_forward(s, 0, D, 1.0, 1.0)
    g = run_backward(s, r, 0, D, 1.0, 1.0)
    torch.cuda.synchronize()
    assert r["amax_n"].item() == 0 and g["amax_dy"].item() == 0
    assert not g["dg_post"].any() and not g["dg_pre"].any() and not g["dgate"].any()


def test_rows_of_zeros_and_of_large_values():
    """eps alone carries a zero row; sums of squares near fp32's range stay finite."""
    M, D = 4, 256
    s = make(M, D, True, 0, True, 10)
    s["x"][0], s["y"][0] = 0.0, 0.0
    s["y"][1], s["x"][1] = 2.0 ** 50, -2.0 ** 50
    r = run_forward(s, M, D, 1.0, 1.0)
    g = run_backward(s, r, M, D, 1.0, 1.0)
    torch.cuda.synchronize()
    check_forward(s, r, 1.0, 1.0)
    check_backward(s, r, g, 1.0, 1.0)
    assert not r["n"][0].any() and r["rstd_post"][0].item() == pytest.approx(EPS ** -0.5, rel=1e-6)


def test_other_stream_and_replayed_graph():
    M, D, a, b = 129, 1024, 1.0, 0.5
    s = make(M, D, True, 1, True, 11)
    side = torch.cuda.Stream()
    want = run_forward(s, M, D, a, b)
    wg = run_backward(s, want, M, D, a, b)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r = run_forward(s, M, D, a, b)
        g = run_backward(s, r, M, D, a, b)
    side.synchronize()
    assert torch.equal(r["n"], want["n"]) and all(torch.equal(g[k], wg[k]) for k in wg)
    # captured, then replayed on changing inputs with eager work in between
    bufs = dict(h=out_rows(M, D), n=out_rows(M, D), r1=torch.empty(M, device="cuda"), r2=torch.empty(M, device="cuda"), dx=out_rows(M, D), dy=out_rows(M, D),
                dgp=torch.empty(D, device="cuda"), dga=torch.empty(1, D, device="cuda"), dgr=torch.empty(D, device="cuda"), am=torch.empty(2, device="cuda"),
                ws=torch.empty(f8.residual_norm_bwd_workspace_bytes(M, D, 1), dtype=torch.uint8, device="cuda"))

    def step():
        f8.residual_norm(s["x"], s["y"], bufs["h"], bufs["n"], s["g_post"], s["gate"], s["g_pre"], a, b, EPS, bufs["r1"], bufs["r2"], bufs["am"][0:1], bufs["ws"])
        f8.residual_norm_bwd(s["y"], bufs["dx"], bufs["dy"], h=bufs["h"], dh=s["dh"], dn=s["dn"], g_post=s["g_post"], gate=s["gate"], g_pre=s["g_pre"],
                             skip_scale=a, branch_scale=b, rstd_post=bufs["r1"], rstd_pre=bufs["r2"], dg_post=bufs["dgp"], dgate=bufs["dga"],
                             dg_pre=bufs["dgr"], amax_dy=bufs["am"][1:2], workspace=bufs["ws"])
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        s["x"].copy_(gen((M, D), 900 + i).cuda()), s["dn"].copy_(gen((M, D), 950 + i, 1e-2).cuda())
        graph.replay()
        torch.cuda.synchronize()
        eager = run_forward(s, M, D, a, b)
        eg = run_backward(s, eager, M, D, a, b)
        torch.cuda.synchronize()
        assert torch.equal(bufs["n"], eager["n"]) and torch.equal(bufs["am"][0:1], eager["amax_n"]) and torch.equal(bufs["am"][1:2], eg["amax_dy"])
        for k, e in (("dx", "dx"), ("dy", "dy"), ("dgp", "dg_post"), ("dga", "dgate"), ("dgr", "dg_pre")):
            assert torch.equal(bufs[k], eg[e]), (i, k)


def test_gradient_against_differences():
    """The GPU's gradients against central differences of the fp64 forward."""
    M, D, a, b = 3, 24, 0.8, 0.7
    s = make(M, D, True, 1, True, 12)
    r = run_forward(s, M, D, a, b)
    g = run_backward(s, r, M, D, a, b)
    torch.cuda.synchronize()
    w = {k: wide(v) for k, v in s.items()}

    def total(v):
        h, _ = ho.residual_h(v["x"], v["y"], v["g_post"], v["gate"], a, b, EPS)
        return (h * w["dh"]).sum() + (ho.norm(h, v["g_pre"], EPS)[0] * w["dn"]).sum()
    pick = np.random.default_rng(0)
    for of, name in (("x", "dx"), ("y", "dy"), ("g_post", "dg_post"), ("gate", "dgate"), ("g_pre", "dg_pre")):
        scale = np.abs(wide(g[name])).max()
        for _ in range(6):
            at = tuple(pick.integers(0, n) for n in w[of].shape)
            up, down = dict(w), dict(w)
            up[of], down[of] = w[of].copy(), w[of].copy()
            up[of][at] += 1e-5
            down[of][at] -= 1e-5
            # h was rounded to bf16 on the GPU: 2^-8 of the terms of t in each, twice, and the result's own rounding
            assert abs((total(up) - total(down)) / 2e-5 - wide(g[name])[at]) <= 4 * HALF * scale, (name, at)


@pytest.mark.parametrize("M,D,gates", [(12, 520, 12), (40, 4096, 2), (2600, 64, 1300), (1100, 256, 1100)])
def test_gradients_on_any_word(M, D, gates):
    """The fp32 results need no more than their own alignment."""
    s = make(M, D, True, gates, True, 13)
    r = run_forward(s, M, D, 1.0, 0.5)
    want = run_backward(s, r, M, D, 1.0, 0.5)
    ws = torch.empty(f8.residual_norm_bwd_workspace_bytes(M, D, gates), dtype=torch.uint8, device="cuda")
    for at in (1, 2, 3):
        flat = torch.full((gates * D + 2 * D + M * 2 + 8 * at + 40,), 5.0, device="cuda")
        dgate, rest = flat[at:at + gates * D].view(gates, D), flat[at + gates * D:]
        dg_post, dg_pre, rstds = rest[1:1 + D], rest[1 + D:1 + 2 * D], rest[1 + 2 * D:1 + 2 * D + 2 * M]
        rstds[:M], rstds[M:] = r["rstd_post"], r["rstd_pre"]
        f8.residual_norm_bwd(s["y"], torch.empty_like(s["y"]), None, h=r["h"], dh=s["dh"], dn=s["dn"], g_post=s["g_post"], gate=s["gate"], g_pre=s["g_pre"],
                             branch_scale=0.5, rstd_post=rstds[:M], rstd_pre=rstds[M:], dg_post=dg_post, dgate=dgate, dg_pre=dg_pre, workspace=ws)
        torch.cuda.synchronize()
        assert torch.equal(dgate, want["dgate"]) and torch.equal(dg_post, want["dg_post"]) and torch.equal(dg_pre, want["dg_pre"])
        assert (flat[:at] == 5.0).all() and rest[0].item() == 5.0 and (rest[1 + 2 * D + 2 * M:] == 5.0).all()


# The backward's kernels that load past the caches, from 2^25 elements on: a wave, and blocks of up to 256, 512 and 1024 threads a row.
@pytest.mark.parametrize("D,post,gates,pre", [(4096, False, 0, True), (8192, True, 8, True), (16384, True, 4, True)]
                         + [(D, post, gates, pre) for D in (512, 1024, 1032, 2816, 4104, 8200) for post in (False, True) for gates in (0, 1)
                            for pre in (False, True)])
def test_large_tensors_have_the_bits_of_their_rows(D, post, gates, pre):
    """Every row of a tensor of more than 2^25 elements has the bits that a call on a part of the rows gives it, which loads the
    other way; the sums over all rows are those over the parts; a part of the first agrees with the oracle."""
    M = ((1 << 25) // D // 64 + 2) * 64
    per_gate, a, b = M // max(gates, 1), 0.75, 1.5
    s = make(0, D, post, gates, pre, 21)
    torch.manual_seed(D)
    for name, std in (("x", 1.0), ("y", 0.5), ("dh", 1e-2), ("dn", 1e-2)):
        if s[name] is not None:
            s[name] = (torch.randn((M, D), device="cuda") * std).bfloat16()
    r = run_forward(s, M, D, a, b)
    g = run_backward(s, r, M, D, a, b)
    torch.cuda.synchronize()

    def rows_of(first, n):
        part = {k: v[first:first + n] if k in ("x", "y", "dh", "dn") and v is not None else v for k, v in s.items()}
        if gates:
            part["gate"] = s["gate"][first // per_gate:first // per_gate + 1]
        pr = run_forward(part, n, D, a, b)
        pg = run_backward(part, pr, n, D, a, b)
        torch.cuda.synchronize()
        rows = slice(first, first + n)
        assert all(v is None or torch.equal(v, r[k][rows]) for k, v in pr.items() if k != "amax_n")
        assert torch.equal(pg["dx"], g["dx"][rows]) and torch.equal(pg["dy"], g["dy"][rows])
        return part, pr, pg
    few = rows_of(0, 40)
    check_forward(*few[:2], a, b)
    check_backward(*few, a, b)
    sums = {k: torch.zeros_like(g[k], dtype=torch.float64) for k in ("dg_post", "dgate", "dg_pre") if g[k] is not None}
    step = per_gate // 4
    for first in range(0, M, step):
        pg = rows_of(first, step)[2]
        for k, v in sums.items():
            (v[first // per_gate] if k == "dgate" else v).add_(pg[k].view(-1).double())
    assert g["amax_dy"].item() == g["dy"].float().abs().max().item()
    if pre:
        assert r["amax_n"].item() == r["n"].float().abs().max().item()
    # The terms are the same fp32 numbers on both sides: only the additions differ, each side's off by the magnitudes' sum times
    # one rounding for each row of a block (256 or more of them), block and group.
    adds = 2 * 2.0 ** -24 * (M / 256 + 66)
    spread = lambda t: t.repeat_interleave(M // len(t), dim=0)
    for k, v in sums.items():
        if k == "dg_pre":
            terms = s["dn"].float() * r["h"].float() * r["rstd_pre"][:, None]
        else:  # t as dx / a, which is off by half a step of bf16
            terms = g["dx"].float() * ((1 + HALF) * b / a) * s["y"].float()
            if post:
                terms *= r["rstd_post"][:, None]
                terms *= s["g_post"].float() if k == "dgate" else 1.0
            terms *= spread(s["gate"].float()) if gates and k == "dg_post" else 1.0
        size = terms.abs().view(gates if k == "dgate" else 1, -1, D).sum(dim=1, dtype=torch.float64).view(v.shape)
        assert ((g[k].double() - v).abs() <= adds * size + 1e-38).all(), k


# a width for each shape of the kernels: rows of a wave with one and two chunks a thread, of up to 256, 512 and 1024 threads, and of two chunks again
@pytest.mark.parametrize("D", (256, 1024, 1032, 2816, 4104, 8200))
@pytest.mark.parametrize("gates", (0, 3))
@pytest.mark.parametrize("post", (False, True))
@pytest.mark.parametrize("pre", (False, True))
def test_every_shape_with_every_form(D, post, gates, pre):
    M, a, b = 21, 0.75, 1.5
    s = make(M, D, post, gates, pre, D)
    r = run_forward(s, M, D, a, b)
    g = run_backward(s, r, M, D, a, b)
    torch.cuda.synchronize()
    check_forward(s, r, a, b)
    check_backward(s, r, g, a, b)
