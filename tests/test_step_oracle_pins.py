"""oracle/step_oracle.py against PyTorch's autograd in fp64, central differences and hand-worked cases (no GPU)."""
import numpy as np
import pytest
import torch

from oracle import step_oracle as so

RNG = lambda seed: np.random.default_rng(seed)


def test_embed_by_hand():
    table = np.arange(12.0).reshape(3, 4)
    out = so.embed([2, -1, 0, 3], table, 0.5)
    assert np.array_equal(out[0], [4, 4.5, 5, 5.5]) and np.array_equal(out[1], np.zeros(4)) and np.array_equal(out[2], [0, 0.5, 1, 1.5])
    assert np.isnan(out[3]).all()
    d, mag, n = so.embed_bwd([2, -1, 2, 3], np.array([[1.0, -2], [9, 9], [4, 1], [9, 9]]), 3, 2.0)
    assert np.array_equal(d, [[0, 0], [0, 0], [10, -2]]) and np.array_equal(mag, [[0, 0], [0, 0], [10, 6]]) and list(n) == [0, 0, 2]


def test_embed_gradient_is_autograds():
    r = RNG(0)
    table, ids, dout = torch.tensor(r.standard_normal((7, 5)), requires_grad=True), torch.tensor(r.integers(0, 7, 20)), torch.tensor(r.standard_normal((20, 5)))
    out = 1.7 * torch.nn.functional.embedding(ids, table)
    out.backward(dout)
    assert np.allclose(so.embed(ids.tolist(), table.detach().numpy(), 1.7), out.detach().numpy(), rtol=1e-14)
    assert np.allclose(so.embed_bwd(ids.tolist(), dout.numpy(), 7, 1.7)[0], table.grad.numpy(), rtol=1e-13, atol=1e-14)


@pytest.mark.parametrize("bias", [False, True])
@pytest.mark.parametrize("add", [False, True])
def test_layernorm_is_torchs(bias, add):
    r = RNG(1)
    h, g, b, dn, dh = (r.standard_normal(s) for s in ((6, 24), 24, 24, (6, 24), (6, 24)))
    th, tg, tb = (torch.tensor(v, requires_grad=True) for v in (h, g, b))
    n = torch.nn.functional.layer_norm(th, (24,), tg, tb if bias else None, 1e-3)
    (n * torch.tensor(dn)).sum().backward()
    got, mean, rstd = so.layernorm(h, g, b if bias else None, 1e-3)
    assert np.allclose(got, n.detach().numpy(), rtol=1e-12, atol=1e-13)
    dx, dg, db = so.layernorm_bwd(h, g, dn, dh if add else None, 1e-3)
    assert np.allclose(dx, th.grad.numpy() + (dh if add else 0), rtol=1e-11, atol=1e-12) and np.allclose(dg, tg.grad.numpy(), rtol=1e-11, atol=1e-12)
    if bias:
        assert np.allclose(db, tb.grad.numpy(), rtol=1e-12, atol=1e-13)


def test_layernorm_gradient_by_differences():
    r = RNG(2)
    h, g, dn = r.standard_normal((2, 8)), r.standard_normal(8), r.standard_normal((2, 8))
    dx, dg, _ = so.layernorm_bwd(h, g, dn, None, 1e-2)
    loss = lambda h, g: (so.layernorm(h, g, None, 1e-2)[0] * dn).sum()
    for i in range(8):
        e = np.zeros((2, 8))
        e[1, i] = 1e-5
        assert abs((loss(h + e, g) - loss(h - e, g)) / 2e-5 - dx[1, i]) < 1e-8
        assert abs((loss(h, g + e[1]) - loss(h, g - e[1])) / 2e-5 - dg[i]) < 1e-8


def test_grad_norm_is_torchs():
    r = RNG(3)
    ts = [r.standard_normal(n) for n in (1, 7, 100)]
    ps = [torch.nn.Parameter(torch.zeros(len(t), dtype=torch.float64)) for t in ts]
    for p, t in zip(ps, ts):
        p.grad = torch.tensor(t)
    norm, total = so.grad_norm(ts)
    assert np.isclose(float(torch.nn.utils.clip_grad_norm_(ps, 0.5)), norm, rtol=1e-14) and np.isclose(total, norm ** 2)
    for p, t in zip(ps, ts):
        assert np.allclose(p.grad.numpy(), t * so.clip_factor(norm, 0.5), rtol=2e-7)
    assert so.grad_norm(ts, True)[0] == max(np.abs(t).max() for t in ts)
    assert np.isnan(so.grad_norm([np.array([1.0, np.nan])], True)[0]) and so.grad_norm([], True) == (0.0, 0.0) and so.grad_norm([])[0] == 0.0


def test_clip_factor():
    assert so.clip_factor(0.0, 1.0) == 1 and so.clip_factor(2.0, 4.0) == 1 and so.clip_factor(np.inf, 1.0) == 0 and np.isnan(so.clip_factor(np.nan, 1.0))
    assert so.clip_factor(4.0, 1.0) == np.float32(1.0) / (np.float32(4.0) + np.float32(1e-6))
