"""Refusals of f8.residual_norm, f8.token_logprobs, f8.distill and their backwards: on the host, before any launch (no GPU)."""
import pytest
import torch

from paper_2410_06511_amd import f8

FAKE = 0x10000  # a 16-byte aligned non-NULL address that is never dereferenced on these paths
NULL, SHAPE, ALIGN, ENUM, WORKSPACE = 1, 2, 3, 4, 5
INF, NAN = float("inf"), float("nan")


def call(f, defaults, **change):
    args = dict(defaults)
    assert set(change) <= set(args)
    args.update(change)
    return getattr(f8.lib(), f)(*args.values())


FORWARD = dict(x=FAKE, ldx=64, y=FAKE, ldy=64, M=5, D=64, g_post=FAKE, gate=FAKE, gate_rows=5, g_pre=FAKE, skip=1.0, branch=1.0, eps=1e-5, h=FAKE, ldh=64,
               n=FAKE, ldn=64, rstd_post=FAKE, rstd_pre=FAKE, amax=FAKE, ws=None, wb=0, stream=None)   # (refused itself: amax without workspace)
BACKWARD = dict(h=FAKE, ldh=64, y=FAKE, ldy=64, dh=FAKE, lddh=64, dn=FAKE, lddn=64, M=5, D=64, g_post=FAKE, gate=FAKE, gate_rows=5, g_pre=FAKE,
                rstd_post=FAKE, rstd_pre=FAKE, skip=1.0, branch=1.0, dx=FAKE, lddx=64, dy=FAKE, lddy=64, dg_post=FAKE, dgate=FAKE, dg_pre=FAKE, amax=FAKE,
                ws=None, wb=0, stream=None)


@pytest.mark.parametrize("status,change", [
    (NULL, dict(x=None)), (NULL, dict(y=None)), (NULL, dict(h=None)), (NULL, dict(n=None)), (NULL, dict(g_pre=None)),
    (NULL, dict(g_post=None)), (NULL, dict(g_pre=None, n=None)), (SHAPE, dict(M=-1)), (SHAPE, dict(M=1 << 31)), (SHAPE, dict(D=60)), (SHAPE, dict(D=-8)),
    (SHAPE, dict(D=16392, ldx=16392, ldy=16392, ldh=16392, ldn=16392)), (SHAPE, dict(gate_rows=2)), (SHAPE, dict(gate_rows=0)), (SHAPE, dict(gate_rows=-1)),
    (SHAPE, dict(gate=None)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=NAN)), (SHAPE, dict(skip=INF)), (SHAPE, dict(branch=NAN)),
    (SHAPE, dict(ldx=56)), (SHAPE, dict(ldy=68)), (SHAPE, dict(ldh=0)), (SHAPE, dict(ldn=63)),
    (ALIGN, dict(x=FAKE + 8)), (ALIGN, dict(n=FAKE + 2)), (ALIGN, dict(g_post=FAKE + 4)), (ALIGN, dict(gate=FAKE + 2)), (ALIGN, dict(g_pre=FAKE + 8)),
    (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE, wb=4096)),
])
def test_residual_norm(status, change):
    assert call("f8_residual_norm", FORWARD, **change) == status


@pytest.mark.parametrize("status,change", [
    (NULL, dict(dn=None)), (NULL, dict(h=None)), (NULL, dict(rstd_pre=None)), (NULL, dict(rstd_post=None)), (NULL, dict(y=None)),
    (NULL, dict(g_pre=None, dn=None)), (NULL, dict(g_pre=None, dn=None, dg_pre=None, dh=None)), (NULL, dict(g_post=None)),
    (NULL, dict(gate=None, gate_rows=0)), (NULL, dict(dy=None)), (NULL, dict(dx=None, dy=None, dg_post=None, dgate=None, dg_pre=None, amax=None)),
    (SHAPE, dict(M=-1)), (SHAPE, dict(D=4)), (SHAPE, dict(gate_rows=3)), (SHAPE, dict(ldh=32)), (SHAPE, dict(ldy=66)), (SHAPE, dict(lddh=8)),
    (SHAPE, dict(lddn=65)), (SHAPE, dict(lddx=60)), (SHAPE, dict(lddy=7)), (SHAPE, dict(skip=NAN)),
    (ALIGN, dict(dy=FAKE + 8)), (ALIGN, dict(dh=FAKE + 8)), (ALIGN, dict(ws=FAKE + 8, wb=1 << 30)), (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE, wb=8192)),
])
def test_residual_norm_bwd(status, change):
    assert call("f8_residual_norm_bwd", BACKWARD, **change) == status


LOGPROBS = dict(z=FAKE, ld=104, M=3, V=100, scale=1.0, targets=FAKE, stats=FAKE, logp=FAKE, entropy=FAKE, k=5, ids=FAKE, top=FAKE, ws=FAKE, wb=1 << 20,
                stream=None)
LOGPROBS_BWD = dict(z=FAKE, ld=104, M=3, V=100, scale=1.0, targets=FAKE, stats=FAKE, entropy=FAKE, d_logp=FAKE, d_entropy=FAKE, dz=FAKE, ldd=104, cols=104,
                    amax=FAKE, ws=FAKE, wb=8192, stream=None)
DISTILL = dict(z=FAKE, ld=104, M=3, V=100, scale=1.0, ids=FAKE, t=FAKE, K=8, tail=0, ts=1.0, targets=FAKE, stats=FAKE, loss=FAKE, logp=FAKE, ws=FAKE,
               wb=1 << 20, stream=None)
DISTILL_BWD = dict(z=FAKE, ld=104, M=3, V=100, scale=1.0, ids=FAKE, t=FAKE, K=8, tail=0, ts=1.0, targets=FAKE, stats=FAKE, d_loss=FAKE, d_logp=FAKE, dz=FAKE,
                   ldd=104, cols=104, amax=FAKE, ws=FAKE, wb=8192, stream=None)
LOGITS = [(NULL, dict(z=None)), (NULL, dict(stats=None)), (SHAPE, dict(M=-1)), (SHAPE, dict(M=1 << 31)), (SHAPE, dict(V=0)), (SHAPE, dict(V=(1 << 22) + 1, ld=1 << 23)),
          (SHAPE, dict(ld=96)), (SHAPE, dict(ld=101)), (SHAPE, dict(scale=0.0)), (SHAPE, dict(scale=-1.0)), (SHAPE, dict(scale=INF)), (SHAPE, dict(scale=NAN)), (SHAPE, dict(scale=3e38)),
          (ALIGN, dict(z=FAKE + 8))]
TEACHER = [(NULL, dict(ids=None)), (NULL, dict(t=None)), (SHAPE, dict(K=0)), (SHAPE, dict(K=129)), (ENUM, dict(tail=2)), (SHAPE, dict(ts=0.0)),
           (SHAPE, dict(ts=NAN)), (SHAPE, dict(tail=1, ts=0.5))]
GRADIENT = [(NULL, dict(dz=None)), (SHAPE, dict(cols=96)), (SHAPE, dict(cols=100)), (SHAPE, dict(ldd=96)), (SHAPE, dict(ldd=108)), (ALIGN, dict(dz=FAKE + 2)),
            (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(wb=4096))]


@pytest.mark.parametrize("status,change", LOGITS + [
    (NULL, dict(logp=None)), (NULL, dict(targets=None)), (NULL, dict(ids=None)), (NULL, dict(top=None)), (SHAPE, dict(k=-1)), (SHAPE, dict(k=129)),
    (SHAPE, dict(V=4)), (WORKSPACE, dict(V=1 << 20, ld=1 << 20, ws=None, wb=0)), (WORKSPACE, dict(V=1 << 20, ld=1 << 20, wb=64)),
    (ALIGN, dict(V=1 << 20, ld=1 << 20, ws=FAKE + 8))])
def test_token_logprobs(status, change):
    assert call("f8_token_logprobs", LOGPROBS, **change) == status


@pytest.mark.parametrize("status,change", LOGITS + GRADIENT + [
    (NULL, dict(targets=None)), (NULL, dict(d_logp=None)), (NULL, dict(entropy=None)), (NULL, dict(targets=None, d_logp=None, d_entropy=None))])
def test_token_logprobs_bwd(status, change):
    assert call("f8_token_logprobs_bwd", LOGPROBS_BWD, **change) == status


@pytest.mark.parametrize("status,change", LOGITS + TEACHER + [(NULL, dict(loss=None)), (NULL, dict(logp=None)), (NULL, dict(targets=None))])
def test_distill(status, change):
    assert call("f8_distill", DISTILL, **change) == status


@pytest.mark.parametrize("status,change", LOGITS + TEACHER + GRADIENT + [(NULL, dict(d_loss=None)), (NULL, dict(d_logp=None)), (NULL, dict(targets=None))])
def test_distill_bwd(status, change):
    assert call("f8_distill_bwd", DISTILL_BWD, **change) == status


def test_workspace_sizes():
    assert f8.logits_workspace_bytes(0, 1000) == 8192 and f8.logits_workspace_bytes(100000, 32768, 20) == 8192   # a row a block
    one = f8.logits_workspace_bytes(1, 131072, 20)
    assert one >= 8192 and one % 256 == 0
    # beyond the columns of one block rows are always shared
    assert f8.logits_workspace_bytes(5000, 1 << 20, 128) >= 5000 * 8 * (16 + 128 * 8)
    assert f8.residual_norm_bwd_workspace_bytes(0, 64) >= 8192
    assert f8.residual_norm_bwd_workspace_bytes(8192, 4096) >= 8192 + 2 * 4096 * 4


def test_binding_refuses_what_the_library_cannot_see():
    """Wrong types, shapes, strides, and tensors that are not on a GPU, are refused before the library is called."""
    bf, M, D, V = torch.bfloat16, 4, 64, 100
    t = lambda *s, dtype=bf: torch.zeros(s, dtype=dtype)
    with pytest.raises(f8.F8Error, match="x: a tensor on the current GPU"):
        f8.residual_norm(t(M, D), t(M, D), t(M, D))
    with pytest.raises(f8.F8Error, match="logits: a tensor on the current GPU"):
        f8.token_logprobs(t(M, 104), V, t(M, 2, dtype=torch.float32))
    with pytest.raises(f8.F8Error, match="a vocabulary of 105 in 104 columns"):
        f8.token_logprobs(t(M, 104), 105, t(M, 2, dtype=torch.float32))
    with pytest.raises(f8.F8Error, match="a gradient of h or of n"):
        f8.residual_norm_bwd(None, t(M, D), None)
    with pytest.raises(f8.F8Error, match="got torch.float32"):
        f8.residual_norm_bwd(None, t(M, D, dtype=torch.float32), None, dh=t(M, D, dtype=torch.float32))
    with pytest.raises(f8.F8Error, match="logits: a tensor on the current GPU"):
        f8.distill(t(M, 104), V, t(M, 3, dtype=torch.int64), t(M, 3, dtype=torch.float32), t(M, 4, dtype=torch.float32), t(M, dtype=torch.float32))


def test_tensors_of_another_device_are_refused(monkeypatch):
    """The library works on the current device: a tensor of another one (stand-ins that say so) is refused."""
    class Elsewhere:
        dtype, shape, device = torch.bfloat16, (4, 64), "cuda:1"
        def get_device(self): return 1
        def stride(self): return (64, 1)
        def is_contiguous(self): return True
        def data_ptr(self): return FAKE
    monkeypatch.setattr(f8, "_device", lambda: 0)
    with pytest.raises(f8.F8Error, match="on cuda:1"):
        f8.residual_norm(Elsewhere(), Elsewhere(), Elsewhere())
    monkeypatch.setattr(f8, "_device", lambda: 1)
    assert f8._rows("x", Elsewhere(), (4, 64), f8._current()) == (FAKE, 64)
    assert f8._packed("x", Elsewhere(), torch.bfloat16, (4, 64), f8._current()) == FAKE


@pytest.mark.parametrize("change,message", [
    (dict(D=16512, Hq=129, Hkv=129, post_norm=True), "up to 16384"), (dict(D=16512, Hq=129, Hkv=129, gate_rows=1), "up to 16384"),
    (dict(D=16512, Hq=129, Hkv=129, branch_scale=0.5), "up to 16384"), (dict(gate_rows=3), "do not divide"), (dict(gate_rows=-1), "do not divide"),
    (dict(gate_rows=64), "do not divide"), (dict(branch_scale=INF), "scale"), (dict(branch_scale=NAN), "scale")])
def test_a_block_refuses_branches_that_its_calls_would(change, message):
    """At its making, before it takes memory, and not at the first call."""
    from paper_2410_06511_amd.block import TransformerBlock
    args = dict(B=2, S=16, D=256, H=256, Hq=2, Hkv=1)
    args.update(change)
    with pytest.raises(AssertionError, match=message):
        TransformerBlock(**args)


@pytest.mark.parametrize("D,gate_rows", [(16, 1 << 60), (16, (1 << 60) + 1), (16384, 1 << 50), (8, (1 << 61) + 8), (0, (1 << 31) + 1)])
def test_gates_whose_size_no_number_holds(D, gate_rows):
    """Without rows every number of gate rows divides them; what the gate then takes must not be counted past 64 bits."""
    shape = dict(M=0, D=D, gate_rows=gate_rows)
    assert call("f8_residual_norm", FORWARD, **shape, ldx=16384, ldy=16384, ldh=16384, ldn=16384) == SHAPE
    assert call("f8_residual_norm_bwd", BACKWARD, **shape, ldh=16384, ldy=16384, lddh=16384, lddn=16384, lddx=16384, lddy=16384) == SHAPE
    assert f8.residual_norm_bwd_workspace_bytes(0, D, gate_rows) == 8192
