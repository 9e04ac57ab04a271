"""f8.layernorm and its backward where a block takes several rows, one after the other: every shape of a row with more rows than the
grid holds and a remainder, loads past the caches, outputs in the place of inputs.  Tolerances of test_gpu_layernorm.py, and for a
mean far from zero a tighter one."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so
from paper_2410_06511_amd import f8
from test_gpu_layernorm import EPS, FP, HALF, backward, check_backward, check_forward, forward, gen, make, wide

pytestmark = pytest.mark.gpu


# Rows of one and two chunks of a wave (four a block, 512 blocks), of a block's thread a chunk (512 blocks up to 3080 columns, 256 from
# there on) and of two chunks a thread: two or three rows for each, some with none left.
@pytest.mark.parametrize("M,D", [(4103, 512), (2051, 1024), (4103, 1000), (1031, 1536), (1031, 2816), (523, 3080), (523, 4096), (523, 4104), (523, 8192), (263, 12288),
                                 (523, 16384)])
def test_backward_of_several_rows_a_block(M, D):
    s = make(M, D, True, True, seed=M % 7)
    r = forward(s, M, D)
    check_forward(s, r)
    for add in (True, False):
        check_backward(s, r, backward(s, r, M, D, add), add)


# With a maximum of n the forward's 2048 blocks go on by the grid's width: rows of a wave (four a block) and of blocks of each size.
@pytest.mark.parametrize("M,D", [(8201, 264), (8203, 1000), (2053, 1536), (2053, 8192), (2053, 16384)])
@pytest.mark.parametrize("residual", [False, True])
def test_forward_with_a_maximum(M, D, residual):
    s = make(M, D, residual, not residual, seed=D % 5)
    r = forward(s, M, D)
    check_forward(s, r)
    rest = forward(s, M, D, amax=False)     # a block a row
    assert all(torch.equal(r[k], rest[k]) for k in ("n", "mean", "rstd"))


# 2^25 elements and more
@pytest.mark.parametrize("M,D", [(65543, 512), (32771, 1024), (21851, 1536), (8195, 4096), (4099, 8192), (2051, 16384)])
def test_backward_past_the_caches(M, D):
    s = make(M, D, False, False)
    r = forward(s, M, D)
    g = backward(s, r, M, D)
    check_backward(s, r, g)
    m = M // 2 + 1     # a row has the same bits in a smaller tensor
    part = {k: v[:m] if v is not None and v.dim() == 2 else v for k, v in s.items()}
    assert torch.equal(backward(part, dict(h=None, mean=r["mean"][:m], rstd=r["rstd"][:m]), m, D)["dx"], g["dx"][:m])


@pytest.mark.parametrize("M,D", [(4103, 512), (1031, 2816), (523, 8192)])
def test_gradients_in_the_place_of_inputs(M, D):
    s = make(M, D, False, True)
    r = forward(s, M, D)
    g = backward(s, r, M, D)
    ws = torch.empty(f8.layernorm_bwd_workspace_bytes(M, D), dtype=torch.uint8, device="cuda")
    for into in ("dn", "dh", "h"):
        u = dict(dn=s["dn"].clone(), dh=s["dh"].clone(), h=s["x"].clone())
        dg, db = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
        f8.layernorm_bwd(u["h"], s["g"], r["mean"], r["rstd"], u["dn"], u[into], u["dh"], dg, db, None, ws)
        assert torch.equal(u[into], g["dx"]) and torch.equal(dg, g["dg"]) and torch.equal(db, g["db"])


@pytest.mark.parametrize("M,D", [(5, 512), (4, 1000), (3, 2816), (3, 8192), (2, 16384)])
def test_a_mean_a_thousand_deviations_away(M, D):
    """Values of 64 and, one in 64, 64.5: multiples of 0.5 whose sums stay below 2^23, so the sum is exact and the mean is off by its
    rounding alone, 2^-24 of it; the differences from it are exact (both lie within a factor of two).  A mean of r deviations costs
    2^-24 r of a deviation, 6e-5 here, beside FP for the sum of squares, the root and the products."""
    x = torch.full((M, D), 64.0)
    for m in range(M):
        x[m, torch.randperm(D, generator=torch.Generator().manual_seed(m))[:D // 64]] = 64.5
    s = dict(x=x.to(torch.bfloat16).cuda(), y=None, g=gen((D,), 1, 0.2, 1.0).cuda(), b=gen((D,), 2, 0.3).cuda(), dn=None, dh=None)
    r = forward(s, M, D)
    h, g, b = wide(s["x"]), wide(s["g"]), wide(s["b"])
    n, mean, rstd = so.layernorm(h, g, b, EPS)
    assert (900 < mean * rstd).all()
    assert (np.abs(wide(r["mean"]) - mean) <= 2.0 ** -24 * mean * (1 + 2.0 ** -20)).all()
    assert (np.abs(wide(r["rstd"]) - rstd) <= FP * rstd).all()
    bound = HALF * np.abs(n) + 2 * FP * np.abs(n - b) + FP * np.abs(b) + np.abs(g) * (rstd * mean * 2.0 ** -24)[:, None]
    assert (np.abs(wide(r["n"]) - n) <= bound).all()
