"""Call sequence from the last block's output to the loss and back, on the C-ABI entry points: final norm, output projection
(a Float8 linear, as the block's), and either of two losses on its logits.

Buffers and the order of calls only: every step runs in the library's kernels.

    x -> rmsnorm -> [Wout] -> logits -> token log probabilities (and entropy), or distillation from a teacher's top entries

The logits' gradient takes the logits' place, and its amax goes with it to the projection's backward, whose cast needs no pass of
its own for it.  The vocabulary need not be a multiple of 16: Wout has `width` rows, those beyond the vocabulary are padding that
takes no part and whose gradients are zero.
"""
import torch

from . import f8


class OutputHead:
    def __init__(self, M, D, vocab, eps=1e-5, scale=1.0, grad_format=f8.E4M3, device="cuda", scaling="dynamic", history_len=16):
        """scale: factor of the logits (an inverse temperature).  M: tokens, as D a multiple of 16."""
        assert scaling in ("dynamic", "delayed")
        self.M, self.D, self.vocab, self.eps, self.scale = M, D, vocab, eps, scale
        N = self.width = (vocab + 15) // 16 * 16
        bf = dict(dtype=torch.bfloat16, device=device)
        f32 = dict(dtype=torch.float32, device=device)
        self.state = f8.ScalingState(f8.DELAYED, history_len, device) if scaling == "delayed" else None
        self.desc = f8.linear_desc(M, D, N, False, grad_format)
        self.saved = f8.Saved(M, D, N, device=device)
        self.ws = f8.new_workspace(max(M, D, N), max(M, D, N), device)
        self.logits_ws = torch.empty(f8.logits_workspace_bytes(M, vocab), dtype=torch.uint8, device=device)
        self.xn, self.rstd, self.a_xn = torch.empty((M, D), **bf), torch.empty(M, **f32), torch.empty(1, **f32)
        self.logits = torch.empty((M, N), **bf)   # from the backward on: their gradient
        self.stats, self.logp, self.entropy = torch.empty((M, 2), **f32), torch.empty(M, **f32), torch.empty(M, **f32)
        self.kd_stats, self.loss = torch.empty((M, 4), **f32), torch.empty(M, **f32)
        self.a_dl = torch.empty(1, **f32)
        self.dxn, self.dx = torch.empty((M, D), **bf), torch.empty((M, D), **bf)
        self.dg, self.dW = torch.empty(D, **f32), torch.empty((N, D), **bf)

    def project(self, x, w, stream=None):
        """w: dict with g [D] and Wout [width, D] (bf16).  Returns the logits [M, width]."""
        s, amax = self, self.state is None
        f8.rmsnorm(x, w["g"], s.eps, s.xn, s.rstd, s.a_xn if amax else None, s.ws, stream)
        if amax:
            f8.linear_fwd_chained(s.desc, s.xn, s.a_xn, w["Wout"], s.logits, None, s.saved, s.ws, stream)
        else:
            f8.linear_fwd_scaled(s.desc, s.state, s.xn, w["Wout"], s.logits, s.saved, s.ws, stream)
        return s.logits

    def forward(self, x, w, targets, entropy=False, stream=None):
        """Log probabilities of the targets [M] (int64; negative: no token); with entropy the distributions' too, in .entropy."""
        self.project(x, w, stream)
        f8.token_logprobs(self.logits, self.vocab, self.stats, targets, self.logp, self.entropy if entropy else None, scale=self.scale,
                          workspace=self.logits_ws, stream=stream)
        return self.logp

    def backward(self, x, w, targets, d_logp, d_entropy=None, stream=None):
        """Gradient of x, from those of .logp and .entropy [M] (next-token training: d_logp = -1 / tokens)."""
        f8.token_logprobs_bwd(self.logits, self.vocab, self.stats, self.logits, targets, None if d_entropy is None else self.entropy, d_logp, d_entropy,
                              self.scale, self.a_dl, self.ws, stream)
        return self._backward(x, w, stream)

    def forward_distill(self, x, w, teacher_ids, teacher_logp, tail=False, teacher_scale=1.0, targets=None, stream=None):
        """Divergence from the teacher's entries [M, K] (f8.token_logprobs of its logits gives them); with targets their log
        probabilities too, in .logp."""
        self.project(x, w, stream)
        f8.distill(self.logits, self.vocab, teacher_ids, teacher_logp, self.kd_stats, self.loss, targets, None if targets is None else self.logp, tail,
                   teacher_scale, self.scale, self.logits_ws, stream)
        return self.loss

    def backward_distill(self, x, w, teacher_ids, teacher_logp, d_loss, tail=False, teacher_scale=1.0, targets=None, d_logp=None, stream=None):
        f8.distill_bwd(self.logits, self.vocab, teacher_ids, teacher_logp, self.kd_stats, self.logits, d_loss, targets, d_logp, tail, teacher_scale,
                       self.scale, self.a_dl, self.ws, stream)
        return self._backward(x, w, stream)

    def _backward(self, x, w, stream):
        s = self
        if s.state is None:
            f8.linear_bwd_chained(s.desc, s.logits, s.a_dl, s.saved, s.dxn, None, s.dW, s.ws, stream)
        else:
            f8.linear_bwd_scaled(s.desc, s.state, s.logits, s.saved, s.dxn, s.dW, s.ws, stream)
        f8.rmsnorm_bwd(x, w["g"], s.rstd, s.dxn, s.dx, s.dg, s.ws, stream)
        return s.dx
