"""Which kernel takes a microscaled product (f8_mx4_gemm.hip): the rule is a function of the sizes, so it is asked without a GPU.  CASES
names a size for every kernel and each of its instances; test_gpu_mx4_products.py runs them, so that a changed estimate cannot
leave a kernel without a test."""
import ctypes as C

import pytest

from paper_2410_06511_amd import f8

KINDS = ("Rows11", "Rows12", "Rows14", "Rows22", "Rows42", "Strip4", "Strip6", "Strip8", "Quarter", "Half", "Full", "FullRows", "FullCols", "Split")


class Plan(C.Structure):
    _fields_ = [("kind", C.c_int), ("ranges", C.c_int), ("whole", C.c_int)]


def plan(M, N, K, workspace_bytes, units=256):
    """(kernel, ranges of the contraction, tiles of the whole rounds)"""
    rule = f8.lib()._ZN2f812plan_productElllmi
    rule.restype, rule.argtypes = Plan, [C.c_int64, C.c_int64, C.c_int64, C.c_size_t, C.c_int]
    p = rule(M, N, K, workspace_bytes, units)
    return KINDS[p.kind], p.ranges, p.whole


# (kernel, ranges, M, N, K): of the tiles one with a contraction of whole groups (and whole ranges), one without; one or several rounds
CASES = [
    ("Rows11", 1, 1, 528, 1040), ("Rows11", 1, 4, 1040, 8192), ("Rows12", 1, 3, 4112, 272), ("Rows12", 1, 17, 528, 1040), ("Rows14", 1, 3, 8208, 528),
    ("Rows22", 1, 4203, 32, 528), ("Rows22", 1, 300, 528, 30000), ("Rows42", 1, 40, 4144, 1040), ("Rows42", 1, 61, 4400, 512),
    ("Strip4", 1, 65, 4176, 512), ("Strip4", 1, 100, 4208, 1040), ("Strip6", 1, 131, 5904, 1536), ("Strip6", 1, 139, 6144, 1120),
    ("Strip8", 1, 206, 6016, 2048), ("Strip8", 1, 195, 5840, 1600), ("Strip8", 1, 1287, 1200, 1568), ("Strip8", 1, 2068, 928, 8192),
    ("Quarter", 1, 2001, 2032, 1024), ("Quarter", 1, 137, 5520, 528), ("Quarter", 1, 5000, 5072, 1024), ("Quarter", 1, 3000, 9040, 528),
    ("Half", 1, 4090, 4080, 512), ("Half", 1, 2999, 1552, 1040), ("Half", 1, 9000, 3056, 512), ("Half", 1, 5001, 5040, 80),
    ("Full", 1, 4090, 4080, 1024), ("Full", 1, 4096, 4096, 1024), ("Full", 1, 2901, 4512, 544), ("Full", 1, 4999, 5104, 1040),
    ("FullRows", 1, 2602, 8000, 1536), ("FullRows", 1, 2600, 8144, 752), ("FullCols", 1, 3872, 5536, 1024), ("FullCols", 1, 8071, 2640, 608),
    ("FullCols", 1, 1939, 18400, 8288),
    ("Split", 4, 2048, 2032, 20480), ("Split", 4, 2001, 2032, 20496), ("Split", 2, 1219, 3328, 32768), ("Split", 2, 526, 6576, 31232),
    ("Split", 2, 1307, 4256, 31600), ("Split", 8, 250, 4000, 60000),
]

# tokens, inputs and outputs of linears, and the kernels of Y, dX and dW: those that a training batch takes, with odd numbers of tokens
LINEARS = [(4090, 1040, 4080, ("Full", "Half", "Half")), (8071, 608, 2640, ("FullCols", "Half", "Strip8")), (2600, 752, 8144, ("FullRows", "Strip8", "Half")),
           (20496, 2048, 2000, ("Full", "Full", "Split"))]


@pytest.mark.parametrize("M,K,N,kinds", LINEARS)
def test_linear(M, K, N, kinds):
    room = f8.mx4_workspace_bytes(M, K, N)
    assert tuple(plan(*s, room)[0] for s in ((M, N, K), (M, K, N), (N, K, M))) == kinds


@pytest.mark.parametrize("kind,ranges,M,N,K", CASES)
def test_kernel(kind, ranges, M, N, K):
    room = f8.mx4_workspace_bytes(M, K, N)
    assert plan(M, N, K, room)[:2] == (kind, ranges)
    if kind == "Split":
        need = 4 * ranges * M * N
        assert need <= room and plan(M, N, K, need)[:2] == (kind, ranges)
        assert plan(M, N, K, need - 1)[0] != "Split" or plan(M, N, K, need - 1)[1] < ranges
        assert plan(M, N, K, 0)[0] != "Split"   # without a workspace it is another kernel's


def test_every_kernel_has_a_size():
    assert {c[0] for c in CASES} == set(KINDS)
    for kind in ("Quarter", "Half", "Full", "FullRows", "FullCols", "Split"):   # both instances: the contraction in whole ranges of whole groups, or not
        whole = [K % 512 == 0 and K // 512 % ranges == 0 for k, ranges, _, _, K in CASES if k == kind]
        assert any(whole) and not all(whole), kind
    assert {r for k, r, _, _, _ in CASES if k == "Split"} == {2, 4, 8}
    rounds = [-(-M // 256) * -(-N // 256) / 256 for k, _, M, N, _ in CASES if k == "Full"]
    assert min(rounds) <= 1 < max(rounds)
    assert any(plan(M, N, K, 0)[2] > 256 for k, _, M, N, K in CASES if k in ("FullRows", "FullCols"))
