"""Every kernel of the microscaled products, at the sizes that test_mx4_rule.py names for it, through f8.mx4_gemm and f8.mx4_linear_*.
Operands are made as codes and scales, so that no cast stands between them and the product, and multiplied in fp64 on the values
that they stand for.

Exact: values of 0, 0.5 and 1 with scales of 1 and 2 in any order, so each product is a multiple of 2^-2 of at most 4, of variance at
most (0.5 x 2.5)^2 = 1.5625.  The sum of any part of up to 60000 of them is below 8 sqrt(60000 x 1.5625) < 2^12 in magnitude (8 deviations,
10^8 sums), and multiples of 2^-2 below 2^12 have 14 bits: what the chip keeps below the largest (13) and fp32 (24) hold them, in
whatever order they are added.  Results have the bits of the exact sum rounded once.
Bounded: any codes, scales of 2^-3 to 2^3; the tolerance of test_gpu_mx4.py."""
import pytest
import torch

from oracle import mx4_oracle as mo
from paper_2410_06511_amd import f8
from test_mx4_rule import CASES, LINEARS, plan

pytestmark = pytest.mark.gpu
BF16, U8, F64 = torch.bfloat16, torch.uint8, torch.float64
GUARD = 4096


def generator(seed):
    g = torch.Generator("cuda")
    g.manual_seed(seed)
    return g


def in_room(t, fill):
    """t's bytes with GUARD bytes of `fill` in front and behind: (a view of t's shape, all of it)"""
    room = torch.full((t.numel() * t.element_size() + 2 * GUARD,), fill, dtype=U8, device="cuda")
    mine = room[GUARD:-GUARD].view(t.dtype).view(t.shape)
    mine.copy_(t)
    return mine, room


def intact(room, fill):
    return bool((room[:GUARD] == fill).all()) and bool((room[-GUARD:] == fill).all())


def placed(scales):
    """scales [rows, blocks] in the order of f8_mx4; bytes of no block 127"""
    rows, nb = scales.shape
    R, groups = (rows + 63) // 64 * 64, (nb + 15) // 16
    whole = torch.full((R, groups * 16), 127, dtype=U8, device="cuda")
    whole[:rows, :nb] = scales
    # [row, group, block / 4 of the group, block % 4] -> [group, row, block % 4, block / 4]
    return whole.view(R, groups, 4, 4).permute(1, 0, 3, 2).contiguous().view(-1)


def values(codes, scales):
    """[rows, blocks * 32] in fp64 of codes [rows, blocks * 32] and scale bytes"""
    grid = torch.tensor(mo.GRID, dtype=F64, device="cuda")
    v = grid[(codes & 7).long()] * torch.where((codes & 8) != 0, -1.0, 1.0).to(F64)
    s = torch.exp2(scales.to(F64) - 127)
    return (v.view(codes.shape[0], -1, 32) * s[:, :, None]).view(codes.shape)


def operand(rows, n, seed, exact):
    """(codes, scale bytes) of [rows, n]: values behind n are zeros"""
    g, nb = generator(seed), (n + 31) // 32
    if exact:
        codes = torch.tensor([0, 1, 2, 9, 10], dtype=U8, device="cuda")[torch.randint(0, 5, (rows, nb * 32), generator=g, device="cuda")]
        scales = torch.randint(127, 129, (rows, nb), generator=g, device="cuda").to(U8)
    else:
        codes = torch.randint(0, 16, (rows, nb * 32), generator=g, device="cuda").to(U8)
        scales = torch.randint(124, 131, (rows, nb), generator=g, device="cuda").to(U8)
    codes[:, n:] = 0
    return codes, scales


def tensor_of(codes, scales, n, fill):
    """An MX4Tensor whose buffers lie among bytes of `fill`: (tensor, rooms)"""
    t = f8.MX4Tensor(codes.shape[0], n, "")
    t.q, qr = in_room(codes[:, 0::2] | (codes[:, 1::2] << 4), fill)
    t.s, sr = in_room(placed(scales), fill)
    t._struct = f8.MX4Struct(t.q.data_ptr(), t.s.data_ptr(), None, None)
    return t, (qr, sr)


def product(a, b, M, N, ws=None):
    """D in a larger matrix of which the rest is left alone"""
    D = torch.full((M + 3, N + 8), 7.0, dtype=BF16, device="cuda")
    f8.mx4_gemm(a, b, D[:M, :N], ws)
    torch.cuda.synchronize()
    assert bool((D[M:] == 7.0).all()) and bool((D[:, N:] == 7.0).all())
    return D[:M, :N]


def workspace(M, K, N, ranges):
    """Exactly what the ranges take, filled with NaN, among guards; none for a kernel without ranges"""
    if ranges == 1:
        return None, None
    return in_room(torch.full((4 * ranges * M * N,), 255, dtype=U8, device="cuda"), 0xA5)


def test_values_and_places_are_the_oracles():
    codes, scales = operand(70, 560, 1, False)
    assert torch.equal(values(codes, scales).cpu(), torch.tensor(mo.values(codes.view(70, -1, 32).cpu().numpy(), scales.cpu().numpy())))
    assert torch.equal(placed(scales).cpu(), torch.tensor(mo.place_scales(scales.cpu().numpy(), 560)))


@pytest.mark.parametrize("kind,ranges,M,N,K", CASES)
def test_kernel(kind, ranges, M, N, K):
    units = torch.cuda.get_device_properties(0).multi_processor_count
    assert plan(M, N, K, 4 * ranges * M * N if ranges > 1 else 0, units)[:2] == (kind, ranges)
    ws, room = workspace(M, K, N, ranges)

    (ca, sa), (cb, sb) = operand(M, K, 1, True), operand(N, K, 2, True)
    exact = (values(ca, sa) @ values(cb, sb).T).to(BF16)     # (fp64 to bf16: one rounding)
    for fill in (0, 255):       # what lies around the operands: zeros, or codes of -6 and scales of NaN
        (a, ra), (b, rb) = tensor_of(ca, sa, K, fill), tensor_of(cb, sb, K, fill)
        D = product(a, b, M, N, ws)
        bad = D != exact
        assert not bad.any().item(), (fill, int(bad.sum()), bad.nonzero()[:4].tolist())
        assert all(intact(r, fill) for r in ra + rb) and (room is None or intact(room, 0xA5))
    del D, exact

    (ca, sa), (cb, sb) = operand(M, K, 3, False), operand(N, K, 4, False)
    va, vb = values(ca, sa), values(cb, sb)
    d, mag = va @ vb.T, va.abs() @ vb.abs().T
    del va, vb
    (a, _), (b, _) = tensor_of(ca, sa, K, 0), tensor_of(cb, sb, K, 0)
    D = product(a, b, M, N, ws)
    bound = 2.0 ** -8 * d.abs() * (1 + 2.0 ** -7) + 2.0 * (K / 8 + 16) * 2.0 ** -24 * mag
    bad = ~((D.to(F64) - d).abs() <= bound)
    assert not bad.any().item(), (int(bad.sum()), bad.nonzero()[:4].tolist())
    if ws is not None:
        ws.fill_(0)
    assert torch.equal(D, product(a, b, M, N, ws))

    # a block that is not a number in one row of each operand: first, last and inner rows and blocks
    nb = sa.shape[1]
    for m, n, at_a, at_b in ((0, N - 1, nb - 1, 0), (M - 1, N // 2, 0, nb - 1), (M // 2, 0, nb // 2, nb // 2)):
        sa_, sb_ = sa.clone(), sb.clone()
        sa_[m, at_a], sb_[n, at_b] = 255, 255
        (a, _), (b, _) = tensor_of(ca, sa_, K, 0), tensor_of(cb, sb_, K, 0)
        E = product(a, b, M, N, ws)
        assert bool(E[m].isnan().all()) and bool(E[:, n].isnan().all())
        E = E.clone()
        E[m], E[:, n] = D[m], D[:, n]
        assert torch.equal(E, D)


@pytest.mark.parametrize("M,K,N,kinds", LINEARS)
def test_linear(M, K, N, kinds):
    g = generator(M)
    X, W, dY = ((torch.randn(s, generator=g, device="cuda") * std).to(BF16) for s, std in (((M, K), 1.0), ((N, K), 0.02), ((M, N), 1e-3)))
    saved, ws = f8.MX4Saved(M, K, N), torch.full((f8.mx4_workspace_bytes(M, K, N),), 255, dtype=U8, device="cuda")
    Y, dX, dW = (torch.full(s, 7.0, dtype=BF16, device="cuda") for s in ((M, N), (M, K), (N, K)))
    f8.mx4_linear_fwd(X, W, Y, saved, ws)
    f8.mx4_linear_bwd(dY, saved, dX, dW, ws)
    torch.cuda.synchronize()

    def decoded(q, s, n):     # the values of codes and placed scales
        rows, nb = q.shape[0], q.shape[1] // 16
        codes = torch.stack((q & 15, q >> 4), dim=2).view(rows, -1)
        scales = s.view(-1, (rows + 63) // 64 * 64, 4, 4).permute(1, 0, 3, 2).reshape((rows + 63) // 64 * 64, -1)[:rows, :nb]
        return values(codes, scales)[:, :n]
    for name, D, a, b in (("Y", Y, decoded(saved.x.q, saved.x.s, K), decoded(saved.w.q, saved.w.s, K)),
                          ("dX", dX, decoded(saved.dy.q, saved.dy.s, N), decoded(saved.w.q_t, saved.w.s_t, N)),
                          ("dW", dW, decoded(saved.dy.q_t, saved.dy.s_t, M), decoded(saved.x.q_t, saved.x.s_t, M))):
        d, mag = a @ b.T, a.abs() @ b.abs().T
        bound = 2.0 ** -8 * d.abs() * (1 + 2.0 ** -7) + 2.0 * (a.shape[1] / 8 + 16) * 2.0 ** -24 * mag + 1e-38
        bad = ~((D.to(F64) - d).abs() <= bound)
        assert not bad.any().item(), (name, int(bad.sum()), bad.nonzero()[:4].tolist())
