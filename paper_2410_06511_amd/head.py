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
        """scale: factor of the logits (an inverse temperature), of every loss.  M: tokens, as D a multiple of 16."""
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

    def projection_stages(self, x, w, stream=None):
        """w: dict with g [D] and Wout [width, D] (bf16).  [(name, call, flops, algorithmic bytes)] in execution order, as the block's."""
        s, M, D = self, self.M, self.D
        if s.state is None:
            norm = lambda: f8.rmsnorm(x, w["g"], s.eps, s.xn, s.rstd, s.a_xn, s.ws, stream)
            linear = lambda: f8.linear_fwd_chained(s.desc, s.xn, s.a_xn, w["Wout"], s.logits, None, s.saved, s.ws, stream)
        else:
            norm = lambda: f8.rmsnorm(x, w["g"], s.eps, s.xn, s.rstd, None, None, stream)
            linear = lambda: f8.linear_fwd_scaled(s.desc, s.state, s.xn, w["Wout"], s.logits, s.saved, s.ws, stream)
        return [("final rmsnorm", norm, 0, 4 * M * D), ("linear Wout fwd", linear, 2 * M * D * s.width, 0)]

    def _backward_stages(self, x, w, loss, stream):
        s, M, D = self, self.M, self.D
        if s.state is None:
            linear = lambda: f8.linear_bwd_chained(s.desc, s.logits, s.a_dl, s.saved, s.dxn, None, s.dW, s.ws, stream)
        else:
            linear = lambda: f8.linear_bwd_scaled(s.desc, s.state, s.logits, s.saved, s.dxn, s.dW, s.ws, stream)
        return [loss, ("linear Wout bwd", linear, 4 * M * D * s.width, 0),
                ("final rmsnorm bwd", lambda: f8.rmsnorm_bwd(x, w["g"], s.rstd, s.dxn, s.dx, s.dg, s.ws, stream), 0, 6 * M * D)]

    def forward_stages(self, x, w, targets, entropy=False, stream=None):
        s = self
        return self.projection_stages(x, w, stream) + [
            ("token log probabilities", lambda: f8.token_logprobs(s.logits, s.vocab, s.stats, targets, s.logp, s.entropy if entropy else None,
                                                                  scale=s.scale, workspace=s.logits_ws, stream=stream), 0, 2 * s.M * s.vocab)]

    def backward_stages(self, x, w, targets, d_logp, d_entropy=None, stream=None):
        s = self
        return self._backward_stages(x, w, (
            "token log probabilities bwd", lambda: f8.token_logprobs_bwd(s.logits, s.vocab, s.stats, s.logits, targets,
                                                                         None if d_entropy is None else s.entropy, d_logp, d_entropy, s.scale, s.a_dl,
                                                                         s.ws, stream), 0, 4 * s.M * s.width), stream)

    def distill_forward_stages(self, x, w, teacher_ids, teacher_logp, tail=False, teacher_scale=1.0, targets=None, stream=None):
        s = self
        return self.projection_stages(x, w, stream) + [
            ("distillation", lambda: f8.distill(s.logits, s.vocab, teacher_ids, teacher_logp, s.kd_stats, s.loss, targets,
                                                None if targets is None else s.logp, tail, teacher_scale, s.scale, s.logits_ws, stream),
             0, 2 * s.M * s.vocab)]

    def distill_backward_stages(self, x, w, teacher_ids, teacher_logp, d_loss, tail=False, teacher_scale=1.0, targets=None, d_logp=None, stream=None):
        s = self
        return self._backward_stages(x, w, (
            "distillation bwd", lambda: f8.distill_bwd(s.logits, s.vocab, teacher_ids, teacher_logp, s.kd_stats, s.logits, d_loss, targets, d_logp, tail,
                                                       teacher_scale, s.scale, s.a_dl, s.ws, stream), 0, 4 * s.M * s.width), stream)

    @staticmethod
    def _run(stages):
        for _, call, _, _ in stages:
            call()

    def project(self, x, w, stream=None):
        """The logits [M, width]."""
        self._run(self.projection_stages(x, w, stream))
        return self.logits

    def forward(self, x, w, targets, entropy=False, stream=None):
        """Log probabilities of the targets [M] (int64; negative: no token); with entropy the distributions' too, in .entropy."""
        self._run(self.forward_stages(x, w, targets, entropy, stream))
        return self.logp

    def backward(self, x, w, targets, d_logp, d_entropy=None, stream=None):
        """Gradient of x, from those of .logp and .entropy [M] (next-token training: d_logp = -1 / tokens)."""
        self._run(self.backward_stages(x, w, targets, d_logp, d_entropy, stream))
        return self.dx

    def forward_distill(self, x, w, teacher_ids, teacher_logp, tail=False, teacher_scale=1.0, targets=None, stream=None):
        """Divergence from the teacher's entries [M, K] (f8.token_logprobs of its logits gives them); with targets their log
        probabilities too, in .logp: under the head's scale, as the divergence, not at temperature 1 beside a softened one."""
        self._run(self.distill_forward_stages(x, w, teacher_ids, teacher_logp, tail, teacher_scale, targets, stream))
        return self.loss

    def backward_distill(self, x, w, teacher_ids, teacher_logp, d_loss, tail=False, teacher_scale=1.0, targets=None, d_logp=None, stream=None):
        self._run(self.distill_backward_stages(x, w, teacher_ids, teacher_logp, d_loss, tail, teacher_scale, targets, d_logp, stream))
        return self.dx
