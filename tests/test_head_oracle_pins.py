"""Pins of oracle/head_oracle.py: autograd in fp64, central differences, closed forms, numpy and torch on the same rows."""
import numpy as np
import pytest
import torch

from oracle import head_oracle as ho

EPS = 1e-5


def rng(seed):
    return np.random.default_rng(seed)


def residual_inputs(seed, M, D, post, gates, pre):
    r = rng(seed)
    return dict(x=r.normal(size=(M, D)), y=r.normal(size=(M, D)), g_post=1 + 0.2 * r.normal(size=D) if post else None,
                gate=r.normal(size=(gates, D)) if gates else None, g_pre=1 + 0.2 * r.normal(size=D) if pre else None,
                dh=r.normal(size=(M, D)), dn=r.normal(size=(M, D)) if pre else None)


@pytest.mark.parametrize("post,gates,pre", [(False, 0, True), (True, 0, True), (True, 1, True), (True, 3, False), (False, 6, True), (False, 1, False)])
def test_residual_against_autograd(post, gates, pre):
    M, D, a, b = 6, 16, 0.9, 0.6
    s = residual_inputs(1, M, D, post, gates, pre)
    t = {k: torch.tensor(v, requires_grad=k[0] != "d") for k, v in s.items() if v is not None}
    norm = lambda v, g: v * torch.rsqrt((v * v).mean(dim=1, keepdim=True) + EPS) * g
    u = norm(t["y"], t["g_post"]) if post else t["y"]
    h = a * t["x"] + b * (t["gate"].repeat_interleave(M // gates, dim=0) * u if gates else u)
    total = (h * t["dh"]).sum()
    want_h, r1 = ho.residual_h(s["x"], s["y"], s["g_post"], s["gate"], a, b, EPS)
    assert np.allclose(want_h, h.detach().numpy(), rtol=1e-13)
    if pre:
        n = norm(h, t["g_pre"])
        total = total + (n * t["dn"]).sum()
        assert np.allclose(ho.norm(want_h, s["g_pre"], EPS)[0], n.detach().numpy(), rtol=1e-13)
    total.backward()
    got = ho.residual_bwd(want_h, s["y"], s["dh"], s["dn"], s["g_post"], s["gate"], s["g_pre"], a, b, EPS)
    for name, of in (("dx", "x"), ("dy", "y"), ("dg_post", "g_post"), ("dgate", "gate"), ("dg_pre", "g_pre")):
        assert (name in got) == (of in t)
        if of in t:
            assert np.allclose(got[name], t[of].grad.numpy(), rtol=1e-11, atol=1e-12), name


def test_logprobs_against_torch_and_differences():
    M, V, scale = 5, 37, 0.7
    r = rng(2)
    z = np.round(r.normal(size=(M, V)) * 3, 1)   # ties
    targets = np.array([0, 36, 5, -1, 7])
    z[1, 3:9] = -np.inf
    got = ho.token_logprobs(z, scale, targets, 9)
    zt = torch.tensor(z)
    lp = torch.log_softmax(zt * scale, dim=1)
    assert np.allclose(got["logp"][[0, 1, 2, 4]], lp[[0, 1, 2, 4], targets[[0, 1, 2, 4]]].numpy(), rtol=1e-13) and got["logp"][3] == 0
    assert np.allclose(scale * got["stats"][:, 0] + got["stats"][:, 1], torch.logsumexp(zt * scale, dim=1).numpy(), rtol=1e-13)
    assert np.allclose(got["entropy"], torch.distributions.Categorical(probs=lp.exp()).entropy().numpy(), rtol=1e-6)
    order = torch.sort(zt, dim=1, descending=True, stable=True).indices[:, :9].numpy()
    assert np.array_equal(got["top_ids"], order)
    d_logp, d_entropy = r.normal(size=M), r.normal(size=M)
    dz = ho.token_logprobs_bwd(z, scale, targets, d_logp, d_entropy)
    f = lambda zz: (lambda o: (np.where(targets >= 0, o["logp"], 0) * d_logp).sum() + (o["entropy"] * d_entropy).sum())(ho.token_logprobs(zz, scale, targets))
    for i, j in [(0, 0), (0, 5), (1, 36), (1, 4), (2, 5), (3, 1), (4, 30)]:
        up, down = z.copy(), z.copy()
        up[i, j] += 1e-5
        down[i, j] -= 1e-5
        assert abs((f(up) - f(down)) / 2e-5 - dz[i, j]) <= 1e-8, (i, j)


def test_rows_with_nothing_and_with_one_entry_left():
    z = np.full((2, 6), -np.inf)
    z[1, 4] = 3.0
    got = ho.token_logprobs(z, 1.0, np.array([2, 4]), 2)
    assert got["logp"].tolist() == [-np.inf, 0.0] and got["entropy"].tolist() == [0.0, 0.0]
    assert got["top_ids"].tolist() == [[0, 1], [4, 0]]
    assert not ho.token_logprobs_bwd(z, 1.0, np.array([2, 4]), np.ones(2), np.ones(2)).any()


@pytest.mark.parametrize("tail", (False, True))
def test_distillation_against_differences_and_autograd(tail):
    M, V, K, scale, ts = 4, 23, 5, 0.8, (1.0 if tail else 1.3)
    r = rng(3)
    z = r.normal(size=(M, V)) * 2
    ids = np.stack([r.permutation(V)[:K] for _ in range(M)])
    ids[1, 2:] = -1
    ids[2, 3] = ids[2, 0]          # twice
    t = np.log(r.dirichlet(np.ones(K), size=M) * 0.8)
    targets, d_loss, d_logp = np.array([3, -1, 5, 22]), r.normal(size=M), r.normal(size=M)
    dz = ho.distill_bwd(z, ids, t, d_loss, scale, tail, ts, targets, d_logp)

    def f(zz):
        lp = ho.token_logprobs(zz, scale, targets)["logp"]
        return (ho.distill(zz, ids, t, scale, tail, ts) * d_loss).sum() + (np.where(targets >= 0, lp, 0) * d_logp).sum()
    for i in range(M):
        for j in list(ids[i][ids[i] >= 0]) + [1, 9, 17]:
            up, down = z.copy(), z.copy()
            up[i, j] += 1e-5
            down[i, j] -= 1e-5
            assert abs((f(up) - f(down)) / 2e-5 - dz[i, j]) <= 1e-8, (i, j)
    # row 0 as a divergence between two distributions
    lp = torch.log_softmax(torch.tensor(z[0]) * scale, dim=0).numpy()
    q = np.exp(t[0]) if tail else np.exp(t[0] * ts) / np.exp(t[0] * ts).sum()
    want = torch.nn.functional.kl_div(torch.tensor(lp[ids[0]]), torch.tensor(q), reduction="sum").item()
    if tail:
        rest = 1 - np.exp(lp[ids[0]]).sum()
        want += (1 - q.sum()) * (np.log(1 - q.sum()) - np.log(rest))
    assert abs(ho.distill(z, ids, t, scale, tail, ts)[0] - want) <= 1e-12


def test_distillation_is_zero_where_the_student_agrees():
    z = rng(4).normal(size=(1, 12))
    lp = ho.token_logprobs(z)["stats"]
    logp = z - lp[:, :1] - lp[:, 1:]
    ids = np.arange(12)[None, :5]
    for cols in (ids, np.arange(12)[None]):
        assert abs(ho.distill(z, cols, logp[:, cols[0]], tail=True)[0]) < 1e-14
        assert np.abs(ho.distill_bwd(z, cols, logp[:, cols[0]], np.ones(1), tail=True)).max() < 1e-14
    none = np.full((1, 3), -1)
    assert ho.distill(z, none, np.zeros((1, 3)))[0] == 0 and not ho.distill_bwd(z, none, np.zeros((1, 3)), np.ones(1)).any()
    assert abs(ho.distill(z, none, np.zeros((1, 3)), tail=True)[0]) < 1e-14


def test_rows_without_entries_have_no_term():
    """The loss is constant there: also with every logit masked, and (without a tail) with entries that all weigh nothing."""
    z = np.random.default_rng(5).normal(size=(3, 9))
    z[1] = -np.inf
    none, zero = np.full((3, 4), -1), np.tile(np.arange(4), (3, 1))
    for ids, t, tail in ((none, np.zeros((3, 4)), False), (none, np.zeros((3, 4)), True), (zero, np.full((3, 4), -np.inf), False)):
        assert not ho.distill(z, ids, t, 0.7, tail).any()
        assert not ho.distill_bwd(z, ids, t, np.ones(3), 0.7, tail).any()


@pytest.mark.parametrize("gap", (0.0, 90.0, 2000.0, 1e30))
def test_a_rest_far_below_the_list_keeps_its_loss_and_gradient(gap):
    """What lies outside the list, as a class of its own, against autograd of the loss written with log sums: also where its
    probability is below every number that fp64 has."""
    r = rng(6)
    z = r.normal(size=(1, 19))
    ids, t = np.array([[3, 7, 11]]), np.log(np.array([[0.3, 0.2, 0.1]]))
    listed = np.isin(np.arange(19), ids)
    z[0, ~listed] -= gap
    scale = 0.7
    zt = torch.tensor(z[0], requires_grad=True)
    total = torch.logsumexp(scale * zt, dim=0)
    rest = scale * zt[torch.tensor(~listed)]
    top = rest.max().detach()   # (torch.logsumexp's gradient is exp(rest - result), which loses log 16 of the result beside 1e30)
    log_rest = top + (rest - top).exp().sum().log() - total
    q = torch.tensor(np.exp(t[0]))
    left = 1 - q.sum()
    loss = (q * (q.log() - (scale * zt[torch.tensor(ids[0])] - total))).sum() + left * (left.log() - log_rest)
    loss.backward()
    assert abs(ho.distill(z, ids, t, scale, True)[0] - loss.item()) <= 1e-13 * (1 + gap)
    dz = ho.distill_bwd(z, ids, t, np.ones(1), scale, True)[0]
    assert np.isfinite(dz).all() and abs(dz[~listed].sum()) > (0.1 if gap else 0.0)
    assert np.abs(dz - zt.grad.numpy()).max() <= 1e-12
