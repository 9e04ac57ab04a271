"""f8.embed and f8.embed_bwd through the C ABI.  The forward is one fp32 product rounded once: its bits are compared.  The
backward's sum of n tokens takes n - 1 additions in fp32 (in pieces, then over them: no more), 2^-24 of the magnitudes each, a
product with the scale, and half a step of the result: 2^-8 of it in bf16, 2^-24 in fp32."""
import numpy as np
import pytest
import torch

import oracle as o
from oracle import step_oracle as so
from paper_2410_06511_amd import f8
from helpers import bits

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def gen(shape, seed, std=1.0):
    g = torch.Generator("cpu")
    g.manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(BF16)


def wide(t):
    return o.bf16_to_f32(bits(t)).astype(np.float64) if t.dtype == BF16 else t.cpu().numpy().astype(np.float64)


def ids_of(kind, M, V, seed=0):
    r = np.random.default_rng(seed + M)
    if kind == "text":       # few often, many rarely, some positions without a token, some ids that there are not
        ids = np.minimum((r.pareto(0.7, M)).astype(np.int64), V - 1)
        ids[r.random(M) < 0.1] = -1
        ids[r.random(M) < 0.02] = V + 5
        return ids
    if kind == "one":        # one token throughout
        return np.full(M, V // 2)
    if kind == "none":
        return np.full(M, -1) if M % 2 else np.full(M, V)
    if kind == "down":       # each once, in falling order
        return (M - 1 - np.arange(M)) % V
    if kind == "two":        # a run that ends with the last token, and tokens without a row
        ids = np.full(M, V - 1)
        ids[::3] = -1
        return ids
    return r.integers(0, V, M)


def backward(ids, dout, V, scale=1.0, dtype=BF16, pitch=0, stream=None):
    M, D = dout.shape
    d = torch.full((V, D + pitch), 7.0, dtype=dtype, device="cuda")[:, :D]
    ws = torch.full((f8.embed_bwd_workspace_bytes(M, V, D),), 255, dtype=torch.uint8, device="cuda")
    if stream is not None:
        torch.cuda.synchronize()   # what was filled above was filled on the current stream
    f8.embed_bwd(ids, dout, d, scale, ws, stream)
    if stream is not None:
        torch.cuda.synchronize()
    return d


def check_backward(d, ids, dout, scale):
    V, half = d.shape[0], 2.0 ** -8 if d.dtype == BF16 else 2.0 ** -24
    ref, mag, n = so.embed_bwd(ids.cpu().tolist(), wide(dout), V, scale)
    assert (np.abs(wide(d) - ref) <= half * np.abs(ref) * (1 + 2.0 ** -7) + 2.0 ** -24 * (n[:, None] + 1) * mag).all()
    assert not wide(d)[n == 0].any()


@pytest.mark.parametrize("M,V,D", [(0, 5, 16), (1, 1, 8), (1, 1000, 4096), (7, 3, 1032), (300, 50, 2816), (5, 20, 16384)])
@pytest.mark.parametrize("scale", [1.0, 53.06599664568480])
def test_forward(M, V, D, scale):
    table, ids = gen((V, D), M + V).cuda(), torch.tensor(ids_of("text", M, V)).cuda()
    if M > 2:
        ids[0], ids[1], ids[2] = -1, V, V - 1
    out = torch.full((M, D), 7.0, dtype=BF16, device="cuda")
    f8.embed(ids, table, out, scale)
    ref = (table[ids.clamp(0, V - 1)].float() * scale).to(BF16)
    ref[ids < 0] = 0
    real = ids < V
    assert torch.equal(out[real].view(torch.int16), ref[real].view(torch.int16)) and bool(out[~real].isnan().all())


def test_forward_with_pitches_and_far_rows():
    """Rows past 2^31 elements of the table; what lies between the rows is left alone."""
    V, D = (1 << 19) + 3, 4096
    table = torch.zeros((V, D + 8), dtype=BF16, device="cuda")[:, :D]
    ids = torch.tensor([V - 1, 0, V - 2, 1 << 18]).cuda()
    table[ids] = gen((4, D), 1).cuda()
    out = torch.full((4, D + 16), 7.0, dtype=BF16, device="cuda")
    f8.embed(ids, table, out[:, :D])
    assert torch.equal(out[:, :D], table[ids]) and bool((out[:, D:] == 7.0).all())


# lengths around the pieces (8 tokens), the sort's groups (64) and chunks (4096), several merges of which the last is uneven
@pytest.mark.parametrize("M", [0, 1, 7, 8, 9, 63, 64, 65, 130, 1000, 4095, 4096, 4097, 8192, 8193, 12289, 20500])
@pytest.mark.parametrize("kind", ["text", "one", "none", "down", "two", "any"])
def test_backward(M, kind):
    V, D = 97, 24
    ids, dout = torch.tensor(ids_of(kind, M, V)).cuda(), gen((M, D), M).cuda()
    check_backward(backward(ids, dout, V), ids, dout, 1.0)


@pytest.mark.parametrize("M,V,D,dtype,scale,pitch", [(300, 5000, 512, BF16, 1.0, 0), (300, 40, 520, F32, 16.0, 24), (65, 1, 2816, BF16, 0.5, 8), (4100, 2, 1024, F32, 1.0, 0),
                                                     (9, 3, 8192, BF16, 90.5, 0), (1, 1000, 4096, F32, 1.0, 8), (2001, 300, 1000, BF16, 1.0, 16)])
def test_backward_sizes_types_and_pitches(M, V, D, dtype, scale, pitch):
    ids = torch.tensor(ids_of("text", M, V)).cuda()
    dout = torch.full((M, D + 2 * pitch), 9.0, dtype=BF16, device="cuda")[:, :D]
    dout[:] = gen((M, D), D).cuda()
    d = backward(ids, dout, V, scale, dtype, pitch)
    check_backward(d, ids, dout, scale)
    if pitch:
        assert bool((d.as_strided((V, D + pitch), (D + pitch, 1))[:, D:] == 7.0).all())


def test_many_tokens_with_longer_pieces():
    M, V, D = 70001, 500, 16
    for kind in ("text", "one"):
        ids, dout = torch.tensor(ids_of(kind, M, V)).cuda(), gen((M, D), 3).cuda()
        a, b = backward(ids, dout, V, dtype=F32), backward(ids, dout, V, dtype=F32)
        check_backward(a, ids, dout, 1.0)
        assert torch.equal(a, b)


def test_whole_numbers_add_up_exactly():
    """The gradient with respect to each position counts once: sums of small whole numbers have no rounding."""
    M, V, D = 9000, 31, 64
    ids, dout = torch.tensor(ids_of("any", M, V)).cuda(), torch.randint(-3, 4, (M, D), generator=torch.Generator().manual_seed(1)).to(BF16).cuda()
    want = torch.zeros((V, D), dtype=torch.float64).index_add_(0, ids.cpu(), dout.cpu().double())
    assert torch.equal(backward(ids, dout, V, dtype=F32).cpu().double(), want)


def test_infinities_stay_in_their_rows():
    ids, dout = torch.tensor([3, 1, 3, 0] * 20).cuda(), gen((80, 32), 5).cuda()
    dout[2, 7], dout[5, 0] = float("inf"), float("nan")
    d = backward(ids, dout, 6)
    assert d[3, 7].item() == float("inf") and d[1, 0].isnan().item()
    d[3, 7] = d[1, 0] = 0
    assert bool(d.isfinite().all())


def test_on_another_stream_and_in_a_graph():
    M, V, D = 5000, 700, 256
    batches = [(torch.tensor(ids_of("text", M, V, i)).cuda(), gen((M, D), i).cuda()) for i in range(3)]
    eager = [backward(ids, dout, V) for ids, dout in batches]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    d = backward(*batches[1], V, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(d, eager[1])
    ids, dout = (t.clone() for t in batches[0])
    table, out, d = gen((V, D), 7).cuda(), torch.empty((M, D), dtype=BF16, device="cuda"), torch.empty((V, D), dtype=BF16, device="cuda")
    ws = torch.empty(f8.embed_bwd_workspace_bytes(M, V, D), dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        f8.embed(ids, table, out)
        f8.embed_bwd(ids, dout, d, workspace=ws)
    for i in (0, 1, 2, 1):
        ids.copy_(batches[i][0]), dout.copy_(batches[i][1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.randn(1 << 20, device="cuda").sum().isfinite().item()
        real = (ids >= 0) & (ids < V)
        assert torch.equal(d, eager[i]) and torch.equal(out[real], table[ids[real]])
