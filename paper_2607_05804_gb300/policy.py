"""The end of a policy model on one packed batch: final norm, LM head, log probabilities of the sampled tokens with their
entropies and alternatives, and the way back -- dL/dlogits, the LM head's and the norm's gradients -- for a policy-gradient
term or an entropy bonus beside the distillation loss.

The norm and everything about the logits run in libturnopd's kernels; the LM head's three products are plain matrix
products, whose results have the head's type: dL/dh too is rounded to it before the norm's backward pass.  A head is made for
one batch: its mask's supervised tokens are counted on the host, and the logits have a row to each.  The gradient is
written over the logits; log probabilities, entropies, alternatives, dgamma and dbeta are the head's own buffers, which the
next call overwrites.
"""
from __future__ import annotations

import torch

from . import (TURNOPD_RMS_NORM, turnopd_norm_bwd, turnopd_norm_bwd_workspace_bytes, turnopd_norm_fwd,
               turnopd_token_logprobs, turnopd_token_logprobs_bwd, turnopd_token_logprobs_workspace_bytes,
               turnopd_turn_stats)


class PolicyHead:
    """gamma, beta [d] (beta or None) and head [vocab, d] are the model's; loss_mask uint8 [T], token_ids int32 [T] the
    batch's.  forward(x) fills logprob, entropy [T] and, for n_top > 0, top_ids, top_logprob [T, n_top]; backward() takes
    dL/dlogprob and dL/dentropy and returns (dx [T, d], dgamma, dbeta, dhead).  Parameters and x may require gradients;
    autograd records nothing of either call."""

    def __init__(self, gamma, head, loss_mask, token_ids, *, beta=None, kind=TURNOPD_RMS_NORM, eps=1e-6, n_top=0):
        self.gamma, self.beta, self.head, self.kind, self.eps, self.n_top = gamma, beta, head, int(kind), float(eps), int(n_top)
        self.loss_mask, self.token_ids = loss_mask, token_ids
        T, (V, d), dev = loss_mask.numel(), head.shape, head.device
        self.at = loss_mask.nonzero()[:, 0]
        n = self.at.numel()
        self.rows = torch.full((T,), -1, dtype=torch.int32, device=dev)
        self.rows[self.at] = torch.arange(n, dtype=torch.int32, device=dev)
        f32 = dict(dtype=torch.float32, device=dev)
        self.h = torch.empty((T, d), dtype=head.dtype, device=dev)
        self.mean, self.rstd = torch.empty(T, **f32), torch.empty(T, **f32)
        self.logits = torch.empty((n, V), dtype=head.dtype, device=dev)
        self.logprob, self.entropy, self.stats = torch.empty(T, **f32), torch.empty(T, **f32), torch.empty((T, 2), **f32)
        self.top_ids = torch.empty((T, n_top), dtype=torch.int32, device=dev) if n_top else None
        self.top_logprob = torch.empty((T, n_top), **f32) if n_top else None
        self.dh = torch.zeros((T, d), dtype=head.dtype, device=dev)
        self.dgamma, self.dbeta = torch.empty(d, **f32), torch.empty(d, **f32) if beta is not None else None
        self.ws_l = torch.empty(max(turnopd_token_logprobs_workspace_bytes(T), 256), dtype=torch.uint8, device=dev)
        self.ws_n = torch.empty(max(turnopd_norm_bwd_workspace_bytes(T, d), 256), dtype=torch.uint8, device=dev)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.ready = False  # the logits are a forward pass's, not yet written over by their gradient

    @torch.no_grad()
    def forward(self, x):
        self.x, self.ready = x, False
        turnopd_norm_fwd(x, self.gamma, self.beta, self.loss_mask, self.kind, self.eps, self.h, self.mean, self.rstd,
                         self.dev_status)
        self.hs = self.h[self.at]
        torch.mm(self.hs, self.head.t(), out=self.logits)
        turnopd_token_logprobs(self.logits, self.logits.shape[1], self.rows, self.token_ids, self.loss_mask, self.n_top,
                               self.logprob, self.entropy, self.stats, self.top_ids, self.top_logprob, self.ws_l,
                               self.dev_status)
        self.ready = True
        return self.logprob, self.entropy

    @torch.no_grad()
    def backward(self, d_logprob, d_entropy=None):
        """Once after each forward pass, with x as it was: after it the logits hold their gradient."""
        if not self.ready:
            raise RuntimeError("PolicyHead.backward needs a forward pass of its own: the logits hold the last one's gradient")
        g = self.logits
        turnopd_token_logprobs_bwd(g, g.shape[1], self.rows, self.token_ids, self.loss_mask, self.stats, self.logprob,
                                   self.entropy, d_logprob, d_entropy, g, 0, self.ws_l, self.dev_status)
        self.ready = False
        dhead = torch.mm(g.t(), self.hs)
        self.dh[self.at] = torch.mm(g, self.head)
        dx = torch.empty_like(self.x)
        turnopd_norm_bwd(self.x, self.gamma, self.loss_mask, self.kind, self.mean, self.rstd, self.dh, dx, self.dgamma,
                         self.dbeta, self.ws_n)
        return dx, self.dgamma, self.dbeta, dhead

    def turn_entropy(self, turn_id, traj_offsets, max_turns):
        """Mean entropy of the supervised tokens at each turn index (0 where no trajectory reaches it)."""
        dev, B = turn_id.device, traj_offsets.numel() - 1
        f64, i32 = dict(dtype=torch.float64, device=dev), dict(dtype=torch.int32, device=dev)
        turn_sum, turn_cnt = torch.empty(max_turns, **f64), torch.empty(max_turns, dtype=torch.int64, device=dev)
        turnopd_turn_stats(self.entropy, turn_id, self.loss_mask, traj_offsets, max_turns,
                           torch.empty(B * max_turns, **f64), torch.empty(B * max_turns, **i32), turn_sum, turn_cnt,
                           torch.empty(max_turns, **i32), self.dev_status)
        return turn_sum / turn_cnt.clamp(min=1)

    def status(self) -> int:
        return int(self.dev_status.item())
