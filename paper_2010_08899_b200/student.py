"""The last stage of a Transformer that is split over workers and learns from a teacher: one training step in which the
packing of DCT and the operators next to it run together, as they would be used.

    hidden --layer norm--> y --DCT-MP pack ... unpack--> y .* M --projection--> logits --distillation--> loss
                                                                  teacher logits --top log-probs----^
    and back: the gradient at y through the same mask, the layer norm's gradients, and every parameter's gradient
    (one flat fp32 vector) through DCT-DP with error feedback at threshold life-span 1, applied by plain SGD.

The worker that holds the layer norm sends ``(cols, vals)``, the teacher sends ``(ids, log-probs)``, the trainer sends
``(idx, val)``: the three messages of the step are the packed ones.  The projection is a library matrix product.
"""
from __future__ import annotations

from typing import NamedTuple, Optional

import torch

from . import binding as B


class StepResult(NamedTuple):
    loss: torch.Tensor          # [rows] fp32, the distillation loss of every row
    sent: torch.Tensor          # the dct_result_t of the gradient's compression (device)
    grad_hidden: torch.Tensor   # [rows, d]: what goes back to the layer below


class Student:
    """Layer norm and projection of ``d`` features to ``vocab`` columns.  The parameters are one flat fp32 vector
    (norm weight, norm bias, projection [vocab, d]); activations have type ``dtype``."""

    def __init__(self, d: int, vocab: int, rows: int, keep: int, top: int, density: float = 0.05, tail: bool = True,
                 temperature: float = 1.0, lr: float = 0.5, dtype=torch.bfloat16, device="cuda", seed: int = 0):
        self.d, self.vocab, self.rows, self.keep, self.top, self.lr = d, vocab, rows, keep, top, lr
        self.mode = B.DCT_DISTILL_TAIL if tail else B.DCT_DISTILL_RENORM
        self.inv_t = 1.0 / temperature
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        n = 2 * d + vocab * d
        new = lambda *shape, dt=torch.float32: torch.empty(*shape, dtype=dt, device=device)
        self.params = torch.zeros(n, device=device)
        self.weight, self.bias = self.params[:d], self.params[d:2 * d]
        self.projection = self.params[2 * d:].view(vocab, d)
        self.weight.fill_(1.0)
        self.projection.copy_(torch.randn(vocab, d, generator=gen, device=device) * d ** -0.5)
        self.grads, self.residual, self.update = torch.zeros(n, device=device), torch.zeros(n, device=device), torch.zeros(n, device=device)
        # what a step needs, laid out once
        self.y, self.y_kept, self.g_kept = new(rows, d, dt=dtype), new(rows, d, dt=dtype), new(rows, d, dt=dtype)
        self.mean, self.rstd, self.loss = new(rows), new(rows), new(rows)
        self.cols, self.vals, self.gvals = new(rows * keep, dt=torch.int16), new(rows * keep, dt=dtype), new(rows * keep, dt=dtype)
        self.ids, self.logprobs = new(rows * top, dt=torch.int32), new(rows * top)
        self.share = torch.full((rows,), 1.0 / rows, device=device)         # the loss is the mean over the rows
        self.k = max(1, int(n * density))
        self.idx, self.val, self.tau = new(self.k, dt=torch.int32), new(self.k), new(1)
        self.sent, self.status, self.applied = (B.new_result(device) for _ in range(3))      # compression, distillation, decompression
        self.norm_ws = B.new_workspace(B.dct_layer_norm_bwd_workspace_bytes(rows, d), device)
        self.send_ws = B.new_workspace(B.dct_dp_select_compress_workspace_bytes(n), device)

    def logits(self, hidden: torch.Tensor) -> torch.Tensor:
        """The student's logits, with the activations that cross the split packed to ``keep`` per row."""
        rows, d = self.rows, self.d
        B.dct_layer_norm_fwd(hidden, rows, d, d, self.weight, self.bias, 1e-5, self.y, d, self.mean, self.rstd)
        B.dct_mp_topk_pack_fwd(self.y, rows, d, d, self.keep, self.cols, self.vals)
        B.dct_mp_unpack(self.cols, self.vals, rows, d, d, self.keep, self.y_kept)
        return self.y_kept @ self.projection.to(self.y.dtype).t()

    def teach(self, teacher_logits: torch.Tensor) -> None:
        """What the teacher sends: the best ``top`` columns of every row with their log-probabilities."""
        B.dct_lm_logprobs_fwd(teacher_logits, self.rows, self.vocab, self.vocab, self.inv_t, None, self.top,
                              top_ids=self.ids, top_logprobs=self.logprobs)

    def step(self, hidden: torch.Tensor, teacher_logits: torch.Tensor) -> StepResult:
        rows, d, vocab = self.rows, self.d, self.vocab
        self.teach(teacher_logits)
        logits = self.logits(hidden)
        # loss, and the gradient in the place of the logits
        B.dct_lm_distill(logits, rows, vocab, vocab, self.inv_t, self.ids, self.logprobs, self.top, self.mode, self.share,
                         self.loss, logits, vocab, self.status)
        torch.mm(logits.t().float(), self.y_kept.float(), out=self.grads[2 * d:].view(vocab, d))
        grad_y = logits @ self.projection.to(logits.dtype)
        # back over the split through the mask of the forward pass
        B.dct_mp_pack_bwd(grad_y, rows, d, d, self.keep, self.cols, self.gvals)
        B.dct_mp_unpack(self.cols, self.gvals, rows, d, d, self.keep, self.g_kept)
        grad_hidden = torch.empty_like(hidden)
        B.dct_layer_norm_bwd(self.g_kept, d, hidden, rows, d, d, self.weight, self.mean, self.rstd, grad_hidden, d,
                             self.grads[:d], self.grads[d:2 * d], self.norm_ws)
        # the trainer's message, and the update it carries
        n = self.params.numel()
        B.dct_dp_select_compress(self.grads, self.residual, n, self.k, self.tau, self.idx, self.val, self.k, self.sent,
                                 self.send_ws)
        B.dct_dp_decompress(self.idx, self.val, self.sent, self.k, self.update, n, False, self.applied)
        self.params.sub_(self.update, alpha=self.lr)
        return StepResult(self.loss, self.sent, grad_hidden)

    def score(self, hidden: torch.Tensor, tokens: torch.Tensor, alternatives: int = 0):
        """Log-probabilities of ``tokens`` (int32, negative: none), entropies and, if asked for, the best alternatives of
        every row: what serving the student returns."""
        rows, vocab = self.rows, self.vocab
        dev = hidden.device
        lp, ent = torch.empty(rows, device=dev), torch.empty(rows, device=dev)
        ids: Optional[torch.Tensor] = torch.empty(rows, alternatives, dtype=torch.int32, device=dev) if alternatives else None
        lps = torch.empty(rows, alternatives, device=dev) if alternatives else None
        B.dct_lm_logprobs_fwd(self.logits(hidden), rows, vocab, vocab, 1.0, tokens, alternatives, lp, ent, None, ids, lps)
        return lp, ent, ids, lps
