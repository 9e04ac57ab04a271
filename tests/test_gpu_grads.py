"""f8.grad_norm and f8.grad_clip through the C ABI.  The squares are exact in fp64 and so, to 2^-40, are their sums: a norm is off
by half a step of fp32, 2^-24.  The scaling is one fp32 product rounded once by a factor that the definition gives in fp32: its
bits are compared."""
import numpy as np
import pytest
import torch

import oracle as o
from oracle import step_oracle as so
from paper_2410_06511_amd import f8
from helpers import bits

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32
STEP = 8192   # elements that a block takes at once


def gen(n, seed, dtype, std=1.0):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return (torch.randn(n, generator=g) * std).to(dtype)


def wide(t):
    return (o.bf16_to_f32(bits(t)) if t.dtype == BF16 else t.cpu().numpy()).astype(np.float64).reshape(-1)


def workspace(lst):
    return torch.full((f8.grad_norm_workspace_bytes(lst),), 255, dtype=torch.uint8, device="cuda")


def norms(tensors, stream=None):
    lst = f8.GradList(tensors)
    norm, total, most = torch.full((1,), 5.0, device="cuda"), torch.full((1,), 5.0, dtype=torch.float64, device="cuda"), torch.full((1,), 5.0, device="cuda")
    ws = workspace(lst), workspace(lst)
    if stream is not None:
        torch.cuda.synchronize()   # what was filled above was filled on the current stream
    f8.grad_norm(lst, norm, total, workspace=ws[0], stream=stream)
    f8.grad_norm(lst, most, kind=f8.NORM_MAX, workspace=ws[1], stream=stream)
    if stream is not None:
        torch.cuda.synchronize()
    return norm, total, most


def check_norms(tensors):
    got = norms(tensors)
    norm, total = so.grad_norm([wide(t) for t in tensors])
    assert abs(got[0].item() - norm) <= 2.0 ** -24 * norm * (1 + 2.0 ** -20) and abs(got[1].item() - total) <= 2.0 ** -40 * total
    assert got[2].item() == so.grad_norm([wide(t) for t in tensors], True)[0]
    return got[0]


def check_clip(tensors, norm, most):
    factor = so.clip_factor(norm.item(), most)
    want = [(t.float().cpu() * float(factor)).to(t.dtype) if factor != 1 else t.cpu() for t in tensors]
    apart = [torch.full_like(t, 7.0) for t in tensors]
    f8.grad_clip(f8.GradList(tensors), norm, most, f8.GradList(apart))
    before = [t.clone() for t in tensors]
    for t, w, b, s in zip(apart, want, before, tensors):
        assert torch.equal(t.cpu(), w) and torch.equal(s, b)
    f8.grad_clip(f8.GradList(tensors), norm, most)
    for t, w in zip(tensors, want):
        assert torch.equal(t.cpu(), w)


SIZES = {
    "one": [1], "few": [7, 8, 9, 0, 1], "steps": [STEP - 1, STEP, STEP + 1, 3 * STEP + 5, 2 * STEP], "many": [(i * 37) % 300 for i in range(250)],
    "block": [6144 * 64, 64 * 64, 64 * 448, 64, 64], "large": [40_000_003, 17_000_000],
    "past the caches": [90_000_007, 50_000_001],
    "launches": [(i * 53) % 9000 + 1 for i in range(600)],
}


@pytest.mark.parametrize("kind", list(SIZES))
@pytest.mark.parametrize("dtypes", ["bf16", "fp32", "both"])
def test_against_the_oracle(kind, dtypes):
    of = lambda i: {"bf16": BF16, "fp32": F32}.get(dtypes, (BF16, F32)[i % 2])
    tensors = [gen(n, i, of(i), 10.0 ** (i % 3 - 3)).cuda() for i, n in enumerate(SIZES[kind])]
    norm = check_norms(tensors)
    for most in (0.37 * norm.item(), 1e30):
        check_clip([t.clone() for t in tensors], norm, most)


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_tensors_on_any_element(dtype):
    """Pieces of one buffer that begin on any element; the source and the result on different ones; what lies around them stays."""
    sizes = [5, 8, 20000, 1, 8193, 31]
    flat, to = gen(sum(sizes) + 40, 1, dtype).cuda(), torch.full((sum(sizes) + 80,), 7.0, dtype=dtype, device="cuda")
    tensors, out, at, of = [], [], 1, 3
    for n in sizes:
        tensors.append(flat[at:at + n]), out.append(to[of:of + n])
        at, of = at + n + 1, of + n + 2
    norm = check_norms(tensors)
    kept = flat.clone()
    f8.grad_clip(f8.GradList(tensors), norm, 1.0, f8.GradList(out))
    factor = float(so.clip_factor(norm.item(), 1.0))
    want = torch.full_like(to, 7.0)
    of = 3
    for t in tensors:
        want[of:of + t.numel()] = (t.float() * factor).to(dtype)
        of += t.numel() + 2
    assert torch.equal(to, want) and torch.equal(flat, kept)
    f8.grad_clip(f8.GradList(tensors), norm, 1.0)
    mask = torch.ones_like(flat, dtype=torch.bool)
    at = 1
    for n in sizes:
        mask[at:at + n] = False
        at += n + 1
    assert torch.equal(flat[mask], kept[mask]) and torch.equal(flat[~mask], (kept[~mask].float() * factor).to(dtype))


def test_magnitudes_whose_squares_leave_fp32():
    for value in (1e-30, 3e30):
        tensors = [torch.full((1000,), value, dtype=F32, device="cuda"), torch.full((24,), value, dtype=BF16, device="cuda")]
        check_norms(tensors)


def test_what_is_not_a_number():
    for bad, where in ((float("nan"), 5), (float("inf"), 70000)):
        for dtype in (BF16, F32):
            tensors = [gen(70001, 1, dtype).cuda(), gen(50, 2, F32).cuda()]
            tensors[0][where] = bad
            norm, total, most = norms(tensors)
            same = lambda v: np.isnan(v) if np.isnan(bad) else v == bad
            assert same(norm.item()) and same(total.item()) and same(most.item())
            f8.grad_clip(f8.GradList(tensors), norm, 1.0)
            if np.isnan(bad):
                assert all(bool(t.isnan().all()) for t in tensors)
            else:   # a factor of zero
                assert not tensors[1].any().item() and tensors[0][where].isnan().item() and not tensors[0][:where].any().item()


def test_an_empty_list_and_a_zero_bound():
    norm, total, most = norms([])
    assert norm.item() == total.item() == most.item() == 0.0
    norm, total, most = norms([torch.empty(0, device="cuda"), torch.zeros(9, dtype=BF16, device="cuda")])
    assert norm.item() == total.item() == most.item() == 0.0
    t = [gen(9, 1, BF16).cuda()]
    norm = check_norms(t)
    f8.grad_clip(f8.GradList(t), norm, 0.0)
    assert not t[0].any().item()


def test_two_lists_share_nothing_and_results_repeat():
    a, b = [gen(3_000_001, 1, BF16).cuda()], [gen(2_000_003, 2, F32).cuda()]
    first = [v.item() for v in norms(a) + norms(b)]
    assert first == [v.item() for v in norms(a) + norms(b)]


def test_on_another_stream_and_in_a_graph():
    sizes = [100_000, 33, 9000]
    batches = [[gen(n, 10 * i + k, (BF16, F32)[k % 2], i + 1.0).cuda() for k, n in enumerate(sizes)] for i in range(3)]
    eager = []
    for ts in batches:
        norm = norms(ts)[0]
        out = [torch.empty_like(t) for t in ts]
        f8.grad_clip(f8.GradList(ts), norm, 2.0, f8.GradList(out))
        eager.append((norm, out))
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = norms(batches[2], side)[0]
    torch.cuda.synchronize()
    assert torch.equal(got, eager[2][0])
    ts = [t.clone() for t in batches[0]]
    lst, norm = f8.GradList(ts), torch.empty(1, device="cuda")
    ws = workspace(lst)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        f8.grad_norm(lst, norm, workspace=ws)
        f8.grad_clip(lst, norm, 2.0)     # in place
    for i in (0, 1, 2, 1):
        for t, b in zip(ts, batches[i]):
            t.copy_(b)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.randn(1 << 20, device="cuda").sum().isfinite().item()
        assert torch.equal(norm, eager[i][0])
        for t, w in zip(ts, eager[i][1]):
            assert torch.equal(t, w)
