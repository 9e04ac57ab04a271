"""Refusals of f8.embed, f8.layernorm, f8.grad_norm and their companions: on the host, before any launch (no GPU)."""
import ctypes as C

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


EMBED = dict(ids=FAKE, M=5, table=FAKE, ldt=64, V=100, D=64, scale=1.0, out=FAKE, ldo=64, stream=None)
EMBED_BWD = dict(ids=FAKE, M=5, dout=FAKE, lddo=64, V=100, D=64, scale=1.0, type=0, dtable=FAKE, ldt=64, ws=None, wb=0, stream=None)
COMMON = [(SHAPE, dict(M=-1)), (SHAPE, dict(M=1 << 31)), (SHAPE, dict(M=(1 << 28) + 1)), (SHAPE, dict(V=-1)), (SHAPE, dict(V=1 << 31)), (SHAPE, dict(D=60)), (SHAPE, dict(D=-8)),
          (SHAPE, dict(D=(1 << 20) + 8)), (SHAPE, dict(scale=INF)), (SHAPE, dict(scale=NAN)), (SHAPE, dict(ldt=56)), (SHAPE, dict(ldt=68)), (NULL, dict(ids=None)),
          (ALIGN, dict(ids=FAKE + 4))]


@pytest.mark.parametrize("status,change", COMMON + [
    (NULL, dict(table=None)), (NULL, dict(out=None)), (SHAPE, dict(ldo=32)), (SHAPE, dict(ldo=65)), (ALIGN, dict(table=FAKE + 8)), (ALIGN, dict(out=FAKE + 2)),
    (SHAPE, dict(M=0x7FFFFFFF, D=1 << 20, ldt=1 << 20, ldo=1 << 20))])
def test_embed(status, change):
    assert call("f8_embed", EMBED, **change) == status


@pytest.mark.parametrize("status,change", COMMON + [
    (NULL, dict(dout=None)), (NULL, dict(dtable=None)), (SHAPE, dict(lddo=32)), (SHAPE, dict(lddo=65)), (ALIGN, dict(dtable=FAKE + 8)), (ALIGN, dict(dout=FAKE + 2)),
    (ENUM, dict(type=2)), (ENUM, dict(type=-1)), (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE, wb=8192)), (ALIGN, dict(ws=FAKE + 8, wb=1 << 30))])
def test_embed_bwd(status, change):
    assert call("f8_embed_bwd", EMBED_BWD, **change) == status


def test_embed_workspace():
    assert f8.embed_bwd_workspace_bytes(0, 100, 64) >= 8192 and f8.embed_bwd_workspace_bytes(-1, 100, 64) == 8192
    for M in (1, 4096, 4097, 1 << 20):   # sorted lists, and no more than the tokens' own gradients for the sums
        size = f8.embed_bwd_workspace_bytes(M, 1000, 512)
        assert 2 * 4 * M <= size <= 8192 + 4 * (4 * M + 256) + (M // 8 + 1) * 2 * 512 * 4


@pytest.mark.parametrize("D", [8, 1024, 4096])
def test_a_workspace_for_the_longest_batch_serves_every_shorter_one(D):
    """Its size grows with the tokens: around the steps of a piece's length (multiples of 1024) and of the lists (4096), and beyond."""
    lengths = [0, 1, 7, 8, 9, 4095, 4096, 4097] + [1024 * i + k for i in range(7, 40) for k in (-1, 0, 1, 500)] + [70001, 1 << 20, (1 << 20) + 1, 1 << 28]
    sizes = [f8.embed_bwd_workspace_bytes(M, 1000, D) for M in lengths]
    assert sizes == sorted(sizes)
    l = f8.lib()
    for longest, M in ((8193, 8192), (10000, 9216), (20000, 8192)):   # (a table without rows: no launch, whose status is a GPU's)
        room = f8.embed_bwd_workspace_bytes(longest, 0, D)
        assert l.f8_embed_bwd(FAKE, M, FAKE, D, 0, D, 1.0, 0, None, D, FAKE, room, None) != WORKSPACE


NORM = dict(x=FAKE, ldx=64, y=FAKE, ldy=64, M=5, D=64, g=FAKE, b=FAKE, eps=1e-5, h=FAKE, ldh=64, n=FAKE, ldn=64, mean=FAKE, rstd=FAKE, amax=FAKE, ws=None, wb=0,
            stream=None)
NORM_BWD = dict(h=FAKE, ldh=64, g=FAKE, mean=FAKE, rstd=FAKE, dn=FAKE, lddn=64, dh=FAKE, lddh=64, M=5, D=64, dx=FAKE, lddx=64, dg=FAKE, db=FAKE, amax=FAKE, ws=None,
                wb=0, stream=None)


@pytest.mark.parametrize("status,change", [
    (NULL, dict(x=None)), (NULL, dict(n=None)), (NULL, dict(g=None)), (NULL, dict(y=None)), (NULL, dict(h=None)), (SHAPE, dict(M=-1)), (SHAPE, dict(M=1 << 31)),
    (SHAPE, dict(D=60)), (SHAPE, dict(D=-8)), (SHAPE, dict(D=16392, ldx=16392, ldy=16392, ldh=16392, ldn=16392)), (SHAPE, dict(eps=-1.0)), (SHAPE, dict(eps=NAN)),
    (SHAPE, dict(eps=INF)), (SHAPE, dict(ldx=56)), (SHAPE, dict(ldy=68)), (SHAPE, dict(ldh=0)), (SHAPE, dict(ldn=63)), (ALIGN, dict(x=FAKE + 8)), (ALIGN, dict(y=FAKE + 8)),
    (ALIGN, dict(h=FAKE + 8)), (ALIGN, dict(n=FAKE + 2)), (ALIGN, dict(g=FAKE + 4)), (ALIGN, dict(b=FAKE + 4)), (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE, wb=4096)),
    (ALIGN, dict(ws=FAKE + 4, wb=8192))])
def test_layernorm(status, change):
    assert call("f8_layernorm", NORM, **change) == status


@pytest.mark.parametrize("status,change", [
    (NULL, dict(h=None)), (NULL, dict(g=None)), (NULL, dict(mean=None)), (NULL, dict(rstd=None)), (NULL, dict(dn=None)), (NULL, dict(dx=None)),
    (NULL, dict(dx=None, dh=None)), (NULL, dict(dx=None, dh=None, amax=None, dg=None, db=None)), (SHAPE, dict(M=-1)), (SHAPE, dict(D=4)), (SHAPE, dict(ldh=32)),
    (SHAPE, dict(lddn=66)), (SHAPE, dict(lddh=8)), (SHAPE, dict(lddx=60)), (ALIGN, dict(dx=FAKE + 8)), (ALIGN, dict(dh=FAKE + 8)), (ALIGN, dict(dn=FAKE + 8)),
    (ALIGN, dict(h=FAKE + 8)), (ALIGN, dict(ws=FAKE + 8, wb=1 << 30)), (WORKSPACE, dict()), (WORKSPACE, dict(ws=FAKE, wb=8192))])
def test_layernorm_bwd(status, change):
    assert call("f8_layernorm_bwd", NORM_BWD, **change) == status


def tensors(*entries):
    return (f8.TensorStruct * len(entries))(*entries)


@pytest.mark.parametrize("status,entry", [(SHAPE, (FAKE, -1, 0)), (SHAPE, (FAKE, (1 << 40) + 1, 0)), (NULL, (None, 3, 0)), (ENUM, (FAKE, 3, 2)), (ENUM, (FAKE, 3, -1)),
                                          (ALIGN, (FAKE + 1, 3, 0)), (ALIGN, (FAKE + 2, 3, 1))])
def test_grad_lists(status, entry):
    bad, good = tensors((FAKE, 8, 1), entry), tensors((FAKE, 8, 1), (FAKE + (1 << 20), entry[1], entry[2]))
    l = f8.lib()
    assert l.f8_grad_norm(bad, 2, 0, FAKE, None, FAKE, 1 << 30, None) == status
    assert l.f8_grad_clip(bad, None, 2, FAKE, 1.0, None) == status and l.f8_grad_clip(tensors((FAKE, 8, 1), (FAKE, 3, 0)), bad, 2, FAKE, 1.0, None) == status
    assert l.f8_grad_norm_workspace_bytes(bad, 2) == 8192 and good is not None


def test_grad_arguments():
    l, t = f8.lib(), tensors((FAKE, 8, 1), (FAKE + 2, 3, 0))
    assert l.f8_grad_norm(None, 2, 0, FAKE, None, FAKE, 1 << 30, None) == NULL and l.f8_grad_norm(t, -1, 0, FAKE, None, FAKE, 1 << 30, None) == SHAPE
    assert l.f8_grad_norm(t, 2, 2, FAKE, None, FAKE, 1 << 30, None) == ENUM and l.f8_grad_norm(t, 2, 0, None, None, FAKE, 1 << 30, None) == NULL
    assert l.f8_grad_norm(t, 2, 0, FAKE, None, None, 0, None) == WORKSPACE and l.f8_grad_norm(t, 2, 0, FAKE, None, FAKE, 4096, None) == WORKSPACE
    assert l.f8_grad_norm(t, 2, 0, FAKE + 2, None, FAKE, 8192, None) == ALIGN and l.f8_grad_norm(t, 2, 0, FAKE, FAKE + 4, FAKE, 8192, None) == ALIGN
    assert l.f8_grad_clip(t, None, 2, None, 1.0, None) == NULL and l.f8_grad_clip(t, None, 2, FAKE, -1.0, None) == SHAPE and l.f8_grad_clip(t, None, 2, FAKE, NAN, None) == SHAPE
    clip = lambda out: l.f8_grad_clip(t, out, 2, FAKE, 1.0, None)
    assert clip(tensors((FAKE, 8, 0), (FAKE + 2, 3, 0))) == ENUM and clip(tensors((FAKE, 7, 1), (FAKE + 2, 3, 0))) == SHAPE
    assert clip(tensors((FAKE + 4, 8, 1), (FAKE + 2, 3, 0))) == SHAPE   # half over its own input


def test_large_lists_have_room_for_every_launch():
    n = 1000
    t = tensors(*[(FAKE, 1 << 34, 0)] * n)
    assert f8.lib().f8_grad_norm_workspace_bytes(t, n) >= 8 * 2048 * (n // 128 + 1)


def test_binding_refuses_what_the_library_cannot_see():
    bf, f32 = torch.zeros((4, 16), dtype=torch.bfloat16), torch.zeros(4)
    for call_ in (lambda: f8.embed(torch.zeros(4, dtype=torch.int64), bf, bf), lambda: f8.embed(torch.zeros(4, dtype=torch.int32), bf, bf),
                  lambda: f8.embed_bwd(torch.zeros(4, dtype=torch.int64), bf, bf), lambda: f8.embed_bwd(torch.zeros(4, dtype=torch.int64), bf, bf.half()),
                  lambda: f8.layernorm(bf, bf[0], bf), lambda: f8.layernorm_bwd(bf, bf[0], f32, f32, bf, bf), lambda: f8.GradList([f32]),
                  lambda: f8.GradList([torch.zeros(4, dtype=torch.float16)])):
        with pytest.raises(f8.F8Error) as e:
            call_()
        assert e.value.code == SHAPE


# ---- microscaled 4-bit linear ------------------------------------------------------------------

MX4 = lambda **change: f8.MX4Struct(*{**dict(q=FAKE, s=FAKE, q_t=FAKE, s_t=FAKE), **change}.values())
QUANTISE = dict(x=FAKE, rows=5, cols=64, ld=64, out=None, stream=None)
GEMM = dict(M=5, N=32, K=64, A=FAKE, sa=FAKE, B=FAKE, sb=FAKE, D=FAKE, ldd=32, ws=None, wb=0, stream=None)


@pytest.mark.parametrize("status,change,codes", [
    (SHAPE, dict(rows=-1), {}), (SHAPE, dict(cols=72, ld=72), {}), (SHAPE, dict(cols=-16), {}), (SHAPE, dict(ld=48), {}), (SHAPE, dict(ld=68), {}), (SHAPE, dict(rows=1 << 23), {}),
    (SHAPE, dict(rows=(1 << 23) - 1, cols=(1 << 23) - 16, ld=1 << 23), {}), (NULL, dict(x=None), {}), (ALIGN, dict(x=FAKE + 8), {}),
    (NULL, {}, dict(q=None)), (NULL, {}, dict(s=None)), (NULL, {}, dict(s_t=None)), (NULL, {}, dict(q=None, s=None, q_t=None, s_t=None)), (ALIGN, {}, dict(q=FAKE + 8)),
    (ALIGN, {}, dict(s_t=FAKE + 4))])
def test_mx4_quantise(status, change, codes):
    t = MX4(**codes)
    assert call("f8_mx4_quantise", QUANTISE, **{"out": C.byref(t), **change}) == status
    assert call("f8_mx4_quantise", QUANTISE) == NULL


@pytest.mark.parametrize("status,change", [
    (SHAPE, dict(M=-1)), (SHAPE, dict(N=24)), (SHAPE, dict(K=-1)), (SHAPE, dict(K=1 << 23)), (SHAPE, dict(ldd=24)), (SHAPE, dict(ldd=36)), (NULL, dict(A=None)), (NULL, dict(sa=None)),
    (NULL, dict(B=None)), (NULL, dict(sb=None)), (NULL, dict(D=None)), (ALIGN, dict(A=FAKE + 8)), (ALIGN, dict(sb=FAKE + 8)), (ALIGN, dict(D=FAKE + 8)), (ALIGN, dict(ws=FAKE + 8, wb=99)),
    (SHAPE, dict(M=(1 << 23) - 1, N=(1 << 23) - 16, ldd=(1 << 23) - 16))])
def test_mx4_gemm(status, change):
    assert call("f8_mx4_gemm", GEMM, **change) == status


@pytest.mark.parametrize("status,change", [(SHAPE, dict(rows=-1)), (SHAPE, dict(cols=12)), (SHAPE, dict(ldo=56)), (NULL, dict(q=None)), (NULL, dict(s=None)), (NULL, dict(out=None)),
                                           (ALIGN, dict(out=FAKE + 8)), (ALIGN, dict(q=FAKE + 8))])
def test_mx4_dequantise(status, change):
    assert call("f8_mx4_dequantise", dict(q=FAKE, s=FAKE, rows=5, cols=64, out=FAKE, ldo=64, stream=None), **change) == status


def test_mx4_linear():
    l = f8.lib()
    def fwd(d=(5, 64, 32), X=FAKE, W=FAKE, Y=FAKE, x=MX4(), w=MX4(), ws=None):
        sv = f8.MX4SavedStruct(x, w, MX4())
        return l.f8_mx4_linear_fwd(C.byref(f8.MX4Desc(*d)), X, W, Y, C.byref(sv), ws, 0, None)
    for d in ((-1, 64, 32), (5, 72, 32), (5, 64, 40), (5, -16, 32), (1 << 23, 64, 32), (5, 1 << 23, 32)):
        assert fwd(d) == SHAPE
    assert fwd(X=None) == NULL and fwd(Y=None) == NULL and fwd(x=MX4(q=None, s=None)) == NULL and fwd(w=MX4(s=None)) == NULL and fwd(w=MX4(q_t=None)) == NULL
    assert fwd(X=FAKE + 2) == ALIGN and fwd(W=FAKE + 8) == ALIGN and fwd(Y=FAKE + 8) == ALIGN and fwd(ws=FAKE + 4) == ALIGN and fwd(x=MX4(q=FAKE + 4)) == ALIGN
    none = dict(q=None, s=None, q_t=None, s_t=None)   # codes of X that are not wanted: of few and short rows only
    assert fwd(x=MX4(**none)) == NULL and fwd((4, 16400, 32), x=MX4(**none)) == NULL and fwd((4, 64, 32), x=MX4(**{**none, "q_t": FAKE, "s_t": FAKE})) == NULL
    assert fwd((4, 64, 32), X=None, x=MX4(**none)) == NULL and fwd((4, 64, 32), X=FAKE + 2, x=MX4(**none)) == ALIGN
    def bwd(d=(5, 64, 32), dY=FAKE, dX=FAKE, dW=FAKE, x=MX4(), w=MX4(), dy=MX4()):
        sv = f8.MX4SavedStruct(x, w, dy)
        return l.f8_mx4_linear_bwd(C.byref(f8.MX4Desc(*d)), dY, C.byref(sv), dX, dW, None, 0, None)
    assert bwd((5, 64, 40)) == SHAPE and bwd(dY=None) == NULL and bwd(dX=None, dW=None) == NULL and bwd(dY=FAKE + 8) == ALIGN and bwd(dW=FAKE + 8) == ALIGN
    assert bwd(dy=MX4(q=None, s=None)) == NULL and bwd(dy=MX4(q_t=None, s_t=None)) == NULL and bwd(x=MX4(q_t=None, s_t=None)) == NULL and bwd(w=MX4(q_t=None, s_t=None)) == NULL
    assert l.f8_mx4_linear_fwd(None, FAKE, FAKE, FAKE, None, None, 0, None) == NULL and l.f8_mx4_linear_bwd(None, FAKE, None, FAKE, FAKE, None, 0, None) == NULL


def test_mx4_sizes():
    assert f8.mx4_scale_bytes(1, 16) == 64 * 16 and f8.mx4_scale_bytes(65, 513) == 2 * 128 * 16 and f8.mx4_scale_bytes(0, 64) == 0 and f8.mx4_scale_bytes(-1, 64) == 0
    assert f8.mx4_workspace_bytes(5, 64, 32) >= 8192 and f8.mx4_workspace_bytes(-1, 64, 32) == 8192
    t = f8.MX4Tensor(5, 48, "qt", "cpu")
    assert t.q.shape == (5, 32) and t.q_t.shape == (48, 16) and t.s.numel() == 64 * 16 and t.s_t.numel() == 64 * 16
    bf = torch.zeros((5, 48), dtype=torch.bfloat16)
    saved = f8.MX4Saved(5, 48, 16, device="cpu")
    for call_ in (lambda: f8.mx4_quantise(bf, t), lambda: f8.mx4_dequantise(t, bf), lambda: f8.mx4_linear_fwd(bf, None, bf, saved), lambda: f8.mx4_gemm(t, t, bf),
                  lambda: f8.mx4_linear_bwd(bf, saved, bf, None), lambda: f8.MX4Saved(6, 48, 16, device="cpu", x=t), lambda: f8.mx4_gemm(t, f8.MX4Tensor(5, 64, "q", "cpu"), bf)):
        with pytest.raises(f8.F8Error) as e:
            call_()
        assert e.value.code == SHAPE
    with pytest.raises(f8.F8Error):
        f8.mx4_linear_bwd(bf, f8.MX4Saved(5, 48, 16, backward=False, device="cpu"), bf, None)
