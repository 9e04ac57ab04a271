"""Call sequence in front of the first block and behind the whole backward, on the C-ABI entry points: token embeddings with their
table's gradient, and the norm of all gradients with its clipping.

Buffers and the order of calls only: every step runs in the library's kernels.

    ids -> rows of the table * scale = x -> blocks -> head;   ... -> dx -> the table's gradient
    gradients of embedding, blocks and head -> their norm -> scaled to a largest norm
"""
import torch

from . import f8


class TokenEmbedding:
    def __init__(self, M, D, vocab, scale=1.0, grad_dtype=torch.bfloat16, device="cuda"):
        """M: tokens; D a multiple of 8.  scale: factor of the embeddings.  grad_dtype: of the table's gradient, bf16 or fp32."""
        assert grad_dtype in (torch.bfloat16, torch.float32)
        self.M, self.D, self.vocab, self.scale = M, D, vocab, scale
        self.out = torch.empty((M, D), dtype=torch.bfloat16, device=device)
        self.dW = torch.empty((vocab, D), dtype=grad_dtype, device=device)
        self.ws = torch.empty(f8.embed_bwd_workspace_bytes(M, vocab, D), dtype=torch.uint8, device=device)

    def gradients(self):
        """Of the weights, as a backward leaves them: what a norm over all gradients takes."""
        return [self.dW]

    def forward_stages(self, ids, w, stream=None):
        """w: dict with Wemb [vocab, D] (bf16).  [(name, call, flops, algorithmic bytes)] in execution order, as the block's."""
        s = self
        return [("embedding", lambda: f8.embed(ids, w["Wemb"], s.out, s.scale, stream), 0, 4 * s.M * s.D)]

    def backward_stages(self, ids, dout, stream=None):
        s = self
        return [("embedding bwd", lambda: f8.embed_bwd(ids, dout, s.dW, s.scale, s.ws, stream), 0, 2 * s.M * s.D + s.dW.nbytes)]

    def forward(self, ids, w, stream=None):
        """The embeddings [M, D] of ids [M] (int64; negative: no token, zeros)."""
        for _, call, _, _ in self.forward_stages(ids, w, stream):
            call()
        return self.out

    def backward(self, ids, dout, stream=None):
        """The table's gradient [vocab, D]: rows without a token are zeros."""
        for _, call, _, _ in self.backward_stages(ids, dout, stream):
            call()
        return self.dW


class GradientClipper:
    """The norm over the gradients of several parts of a model (each with a gradients() of its own) and their scaling in place."""

    def __init__(self, parts, most, kind=f8.NORM_2, device="cuda"):
        """most: the largest norm that is left as it is.  kind: f8.NORM_2, or f8.NORM_MAX for the largest magnitude."""
        self.grads = f8.GradList([g for p in parts for g in p.gradients()])
        self.most, self.kind = most, kind
        self.norm = torch.empty(1, dtype=torch.float32, device=device)
        self.ws = torch.empty(f8.grad_norm_workspace_bytes(self.grads), dtype=torch.uint8, device=device)

    def stages(self, stream=None):
        s, size = self, sum(g.nbytes for g in self.grads.tensors)
        return [("gradient norm", lambda: f8.grad_norm(s.grads, s.norm, kind=s.kind, workspace=s.ws, stream=stream), 0, size),
                ("clipping", lambda: f8.grad_clip(s.grads, s.norm, s.most, stream=stream), 0, 2 * size)]

    def clip(self, stream=None):
        """Scales the gradients and returns their norm before that, on the GPU."""
        for _, call, _, _ in self.stages(stream):
            call()
        return self.norm
