"""The operators of a training step as a step uses them: blocks and an output head with layer norms, token embeddings in front, a
microscaled projection, and the norm of all gradients behind.  Every operator's outputs are compared with oracle/ on the tensors
that it read in the run itself, with the tolerances of the operators' own tests; whole steps are replayed from a graph."""
import pytest
import torch

from oracle import mx4_oracle as mo
from oracle import step_oracle as so
from paper_2410_06511_amd import f8
from paper_2410_06511_amd.block import TransformerBlock
from paper_2410_06511_amd.embedding import GradientClipper, TokenEmbedding
from paper_2410_06511_amd.head import OutputHead
import test_gpu_embed as te
import test_gpu_grads as tg
import test_gpu_layernorm as tn
import test_gpu_logits as tl
import test_gpu_mx4 as tm
from test_gpu_layer import gen

pytestmark = pytest.mark.gpu

BF16, EPS = torch.bfloat16, 1e-5


def weights(D, H, Hq, Hkv, hd, seed, bias):
    w = {"g1": gen((D,), seed, 0.3) + 1, "g2": gen((D,), seed + 1, 0.3) + 1, "Wqkv": gen(((Hq + 2 * Hkv) * hd, D), seed + 2, 0.04),
         "Wo": gen((D, D), seed + 3, 0.04), "W13": gen((2 * H, D), seed + 4, 0.04), "W2": gen((D, H), seed + 5, 0.04)}
    if bias:
        w.update(b1=gen((D,), seed + 6, 0.2), b2=gen((D,), seed + 7, 0.2))
    return {k: v.bfloat16().cuda() for k, v in w.items()}


def tokens(M, V, seed):
    ids = te.ids_of("text", M, V, seed)
    ids[ids >= V] = -1    # (an id that the table has not is the operator's own test)
    return torch.tensor(ids).cuda()


def same(a, b):
    return torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def largest(t):
    return t.float().abs().max().reshape(1)


@pytest.mark.parametrize("scaling", ("dynamic", "delayed"))
@pytest.mark.parametrize("bias", (False, True))
def test_block_of_layer_norms(bias, scaling):
    B, S, Hq, Hkv, hd, H = 2, 136, 4, 2, 128, 512
    D, M = Hq * hd, B * S
    w = weights(D, H, Hq, Hkv, hd, 100, bias)
    x, dout = gen((M, D), 1).cuda(), gen((M, D), 2, 1e-2).cuda()
    blk = TransformerBlock(B, S, D, H, Hq, Hkv, hd, EPS, scaling=scaling, norm="layer", norm_bias=bias)
    for _ in range(2 if scaling == "delayed" else 1):
        blk.forward(x, w)
        blk.backward(x, w, dout)
    torch.cuda.synchronize()
    dynamic = scaling == "dynamic"
    s1 = dict(x=x, y=None, g=w["g1"], b=w.get("b1"), dn=blk.dxn, dh=blk.dh1)
    r1 = dict(h=None, n=blk.xn, mean=blk.mean1, rstd=blk.rstd1, amax=blk.a_xn if dynamic else None)
    s2 = dict(x=x, y=blk.yo, g=w["g2"], b=w.get("b2"), dn=blk.dhn, dh=dout)
    r2 = dict(h=blk.h1, n=blk.hn, mean=blk.mean2, rstd=blk.rstd2, amax=blk.a_hn if dynamic else None)
    tn.check_forward(s1, r1), tn.check_forward(s2, r2)
    none = torch.tensor(tn.wide(s1["dn"]).sum(axis=0)), torch.tensor(tn.wide(s2["dn"]).sum(axis=0))   # (a block without biases has no db)
    tn.check_backward(s1, r1, dict(dx=blk.dx, dg=blk.dg1, db=blk.db1 if bias else none[0], amax=largest(blk.dx)))
    tn.check_backward(s2, r2, dict(dx=blk.dh1, dg=blk.dg2, db=blk.db2 if bias else none[1], amax=blk.a_bwd[0:1] if dynamic else largest(blk.dh1)))
    assert torch.equal(blk.out, (blk.h1.float() + blk.y2.float()).to(BF16))
    # the linears behind the norms took them and their amax: the same calls on their own
    if dynamic:
        datt, dWo = torch.empty_like(blk.datt), torch.empty_like(blk.dWo)
        f8.linear_bwd(blk.d_o, blk.dh1, blk.s_o, datt, dWo, blk.ws)
        torch.cuda.synchronize()
        assert same(datt, blk.datt) and same(dWo, blk.dWo)


@pytest.mark.parametrize("scaling", ("dynamic", "delayed"))
@pytest.mark.parametrize("recompute", (True, "selective"))
def test_block_of_layer_norms_recomputes_its_own_bits(scaling, recompute):
    B, S, Hq, Hkv, hd, H = 1, 272, 2, 1, 128, 512
    D, M = Hq * hd, B * S
    w = weights(D, H, Hq, Hkv, hd, 200, True)
    x, dout = gen((M, D), 11).cuda(), gen((M, D), 12, 1e-2).cuda()
    kept, redo = (TransformerBlock(B, S, D, H, Hq, Hkv, hd, scaling=scaling, norm="layer", norm_bias=True) for _ in range(2))
    for _ in range(2):
        kept.forward(x, w)
        kept.backward(x, w, dout)
        redo.forward(x, w)
        for n in ("xn", "h1", "hn", "mean1", "rstd1", "mean2", "rstd2") + (("yo", "att") if recompute is True else ()):
            getattr(redo, n).fill_(5.0)
        redo.backward(x, w, dout, recompute=recompute)
        torch.cuda.synchronize()
        for n in ("dx", "dWqkv", "dWo", "dW13", "dW2", "dg1", "dg2", "db1", "db2"):
            assert same(getattr(kept, n), getattr(redo, n)), n


def test_what_a_block_and_a_head_refuse():
    for made in (lambda: TransformerBlock(1, 128, 256, 256, 2, 1, norm="batch"), lambda: TransformerBlock(1, 128, 256, 256, 2, 1, norm_bias=True),
                 lambda: TransformerBlock(1, 128, 256, 256, 2, 1, norm="layer", post_norm=True), lambda: TransformerBlock(1, 128, 256, 256, 2, 1, norm="layer", gate_rows=1),
                 lambda: OutputHead(16, 64, 100, norm="batch"), lambda: OutputHead(16, 64, 100, norm_bias=True), lambda: OutputHead(16, 16400, 100, norm="layer")):
        with pytest.raises(AssertionError):
            made()
    blk = TransformerBlock(1, 128, 256, 256, 2, 1)
    assert not any(hasattr(blk, n) for n in ("mean1", "db1", "ln_ws")) and len(blk.gradients()) == 6
    # a gradient that is listed twice would be scaled twice, or by chance once
    t = torch.zeros(64, device="cuda")
    for twice in ([t, t], [t[:32], t[31:]], [t[8:9], t[:0], t]):
        with pytest.raises(f8.F8Error) as e:
            f8.GradList(twice)
        assert e.value.code == f8.F8_ERR_SHAPE
    assert len(f8.GradList([t[:32], t[32:], t[5:5], t[5:5]])) == 4


@pytest.mark.parametrize("scaling", ("dynamic", "delayed"))
def test_a_whole_step(scaling):
    """Embeddings, two blocks, the head, back, and clipping: every new operator against the oracle on what it read, and the step
    replayed from a graph with the bits of an eager one."""
    B, S, Hq, Hkv, hd, H, V = 2, 136, 2, 1, 128, 512, 1003
    D, M, most = Hq * hd, B * S, 0.25
    embedding = TokenEmbedding(M, D, V, scale=D ** 0.5)
    blocks = [TransformerBlock(B, S, D, H, Hq, Hkv, hd, EPS, scaling=scaling, norm="layer", norm_bias=True) for _ in range(2)]
    head = OutputHead(M, D, V, EPS, scaling=scaling, norm="layer", norm_bias=True)
    clipper = GradientClipper([embedding, *blocks, head], most)
    we = {"Wemb": gen((V, D), 7, 1 / 16).cuda()}
    ws = [weights(D, H, Hq, Hkv, hd, 300 + 50 * i, True) for i in range(2)]
    wh = {"g": (gen((D,), 8, 0.2) + 1).bfloat16().cuda(), "b": gen((D,), 9, 0.2).cuda(), "Wout": gen((head.width, D), 10, 0.05).cuda()}
    batches = [(tokens(M, V, i), tl.make_targets(M, V, 11 + i)) for i in range(3)]
    ids, targets = (t.clone() for t in batches[0])
    d_logp = torch.full((M,), -1.0 / M, device="cuda")
    before = []

    def step(stop=False):
        h = embedding.forward(ids, we)
        for b, w in zip(blocks, ws):
            h = b.forward(h, w)
        head.forward(h, wh, targets)
        d = head.backward(h, wh, targets, d_logp)
        for b, w, x in zip(blocks[::-1], ws[::-1], (blocks[0].out, embedding.out)):
            d = b.backward(x, w, d)
        embedding.backward(ids, d)
        if not stop:
            clipper.clip()

    for _ in range(2):   # (the first delayed step casts with scales of 1)
        step(stop=True)
    torch.cuda.synchronize()
    before = [t.clone() for t in clipper.grads.tensors]
    # embeddings
    ref = (we["Wemb"][ids.clamp(0, V - 1)].float() * torch.tensor(D ** 0.5)).to(BF16)
    ref[ids < 0] = 0
    assert torch.equal(embedding.out, ref)
    te.check_backward(embedding.dW, ids, blocks[0].dx, D ** 0.5)
    # the head's norm
    s = dict(x=blocks[1].out, y=None, g=wh["g"], b=wh["b"], dn=head.dxn, dh=None)
    r = dict(h=None, n=head.xn, mean=head.mean, rstd=head.rstd, amax=head.a_xn if scaling == "dynamic" else None)
    tn.check_forward(s, r), tn.check_backward(s, r, dict(dx=head.dx, dg=head.dg, db=head.db, amax=largest(head.dx)), add=False)
    # the norm of everything, and the scaling
    clipper.clip()
    torch.cuda.synchronize()
    norm, _ = so.grad_norm([tg.wide(t) for t in before])
    assert abs(clipper.norm.item() - norm) <= 2.0 ** -24 * norm * (1 + 2.0 ** -20) and norm > most
    factor = float(so.clip_factor(clipper.norm.item(), most))
    assert len(before) == 1 + 2 * 8 + 3
    for t, b in zip(clipper.grads.tensors, before):
        assert torch.equal(t, (b.float() * factor).to(t.dtype))
    # replays: under dynamic scaling a step depends on its inputs alone
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    results = lambda: [t.clone() for t in (head.logp, clipper.norm, *clipper.grads.tensors)]
    for i in (1, 2, 0, 1):
        ids.copy_(batches[i][0]), targets.copy_(batches[i][1])
        graph.replay()
        torch.cuda.synchronize()
        got = results()
        assert torch.isfinite(got[1]).all() and torch.randn(1 << 20, device="cuda").sum().isfinite().item()
        if scaling == "dynamic":
            step()
            torch.cuda.synchronize()
            assert all(same(a, b) for a, b in zip(got, results())), i
        total = torch.stack([t.double().square().sum() for t in got[2:]]).sum().sqrt().item()
        assert total <= most * 1.01   # (each of the gradients was rounded once more)


def test_microscaled_projection_in_a_step():
    """ids -> embeddings -> layer norm with a residual -> microscaled linear -> log probabilities, back, and clipping, captured
    with one workspace for everything that takes one."""
    M, D, V = 200, 528, 1040
    table, y = gen((V, D), 1, 0.05).cuda(), gen((M, D), 2, 0.3).cuda()
    g, b, W = (gen((D,), 3, 0.2) + 1).bfloat16().cuda(), gen((D,), 4, 0.2).cuda(), gen((V, D), 5, 0.05).cuda()
    batches = [(tokens(M, V, i), tl.make_targets(M, V, 20 + i)) for i in range(3)]
    ids, targets = (t.clone() for t in batches[0])
    d_logp = torch.full((M,), -1.0 / M, device="cuda")
    new = lambda *s, dtype=BF16: torch.empty(s, dtype=dtype, device="cuda")
    f32 = lambda *s: new(*s, dtype=torch.float32)
    t = dict(x=new(M, D), h=new(M, D), n=new(M, D), mean=f32(M), rstd=f32(M), z=new(M, V), stats=f32(M, 2), logp=f32(M), dz=new(M, V), dn=new(M, D), dx=new(M, D),
             dW=new(V, D), dg=f32(D), db=f32(D), dtable=f32(V, D), norm=f32(1), amax=f32(1))
    saved = f8.MX4Saved(M, D, V)
    grads = f8.GradList([t[k] for k in ("dW", "dg", "db", "dtable")])
    sizes = (f8.mx4_workspace_bytes(M, D, V), f8.logits_workspace_bytes(M, V), f8.layernorm_bwd_workspace_bytes(M, D), f8.embed_bwd_workspace_bytes(M, V, D),
             f8.grad_norm_workspace_bytes(grads))
    ws = new(max(sizes), dtype=torch.uint8)

    def forward_backward():
        f8.embed(ids, table, t["x"], 4.0)
        f8.layernorm(t["x"], g, t["n"], b, y, t["h"], EPS, t["mean"], t["rstd"])
        f8.mx4_linear_fwd(t["n"], W, t["z"], saved, ws)
        f8.token_logprobs(t["z"], V, t["stats"], targets, t["logp"], workspace=ws)
        f8.token_logprobs_bwd(t["z"], V, t["stats"], t["dz"], targets, d_logp=d_logp, workspace=ws)
        f8.mx4_linear_bwd(t["dz"], saved, t["dn"], t["dW"], ws)
        f8.layernorm_bwd(t["h"], g, t["mean"], t["rstd"], t["dn"], t["dx"], None, t["dg"], t["db"], t["amax"], ws)
        f8.embed_bwd(ids, t["dx"], t["dtable"], 4.0, ws)

    def clip():
        f8.grad_norm(grads, t["norm"], workspace=ws)
        f8.grad_clip(grads, t["norm"], 0.01)

    forward_backward()
    torch.cuda.synchronize()
    s = dict(x=t["x"], y=y, g=g, b=b, dn=t["dn"], dh=None)
    r = dict(h=t["h"], n=t["n"], mean=t["mean"], rstd=t["rstd"], amax=None)
    tn.check_forward(s, r), tn.check_backward(s, r, t, add=False)
    n, w, dz = tm.wide(t["n"]), tm.wide(W), tm.wide(t["dz"])
    tm.check_product(t["z"], mo.rounded(n), mo.rounded(w), "z")
    tm.check_product(t["dn"], mo.rounded(dz), mo.rounded(w.T), "dn")
    tm.check_product(t["dW"], mo.rounded(dz.T), mo.rounded(n.T), "dW")
    te.check_backward(t["dtable"], ids, t["dx"], 4.0)
    norm = tg.check_norms(grads.tensors)
    tg.check_clip(grads.tensors, norm, 0.01)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        forward_backward(), clip()
    keys = ("logp", "norm", "dW", "dg", "db", "dtable", "amax")
    for i in (1, 2, 0, 1):
        ids.copy_(batches[i][0]), targets.copy_(batches[i][1])
        for k in keys:
            t[k].fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        got = {k: t[k].clone() for k in keys}
        ws.fill_(255)
        forward_backward(), clip()
        torch.cuda.synchronize()
        assert all(same(got[k], t[k]) for k in keys), i
