"""A policy model from its token ids to the hidden states in front of the final norm, and the way back: embedding, blocks, and
between the blocks their norms, gates and residual connections.  With policy.PolicyHead behind it that is the whole model.

Everything outside of the blocks runs in libturnopd's kernels.  A block is any callable [T, d] -> [T, d]; it runs without a
record in the forward pass and once more, from the input that was kept, in the backward pass, where autograd gives its
gradients.  It may not write into its input, nor into an output that it gave before.  What it draws from torch's default
generators it draws again the second time (a forward pass captured into a CUDA graph cannot keep their states: backward refuses
blocks that draw then); on anything else that changes between its two runs -- a generator of its own, running statistics -- its
result may not depend.  It runs under the autocast that is on around forward, in both runs.

What is kept in between -- each block's input and output and the residual stream after it -- can be kept in 8 bits
(turnopd_act8_store): 1.03 bytes an element instead of two or four, at the price of the codes' rounding in the gradients.
"""
from __future__ import annotations

from contextlib import nullcontext
from dataclasses import dataclass
from typing import Any

import torch

from . import (TURNOPD_ACCUMULATE_GRAD, TURNOPD_RMS_NORM, turnopd_act8_load, turnopd_act8_store, turnopd_block_norm_bwd,
               turnopd_block_norm_bwd_workspace_bytes, turnopd_block_norm_fwd, turnopd_embedding_bwd,
               turnopd_embedding_bwd_workspace_bytes, turnopd_embedding_fwd, turnopd_norm_fwd)

CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}


class _Generators:
    """The states of torch's default generators, on the host and on one device, when it was made.  As a context: them again,
    and afterwards those that it found."""

    def __init__(self, device):
        self.device, self.states = device, (torch.get_rng_state(), torch.cuda.get_rng_state(device))

    def _set(self, states):
        torch.set_rng_state(states[0])
        torch.cuda.set_rng_state(states[1], self.device)

    def __enter__(self):
        self.found = _Generators(self.device).states
        self._set(self.states)

    def __exit__(self, *_):
        self._set(self.found)


class _Autocast:
    """Autocast as it was when this was made.  Without its cache: what it casts of a parameter in the forward pass, where nothing
    is recorded, would be taken for the backward pass's, and the parameter would have no gradient."""

    def __init__(self):
        self.on, self.dtype = torch.is_autocast_enabled("cuda"), torch.get_autocast_dtype("cuda")

    def __call__(self):
        if not self.on and not torch.is_autocast_enabled("cuda"):
            return nullcontext()
        return torch.autocast("cuda", dtype=self.dtype, enabled=self.on, cache_enabled=False)


class _NoDraws:
    """A context that draws nothing from torch's default generators, or raises."""

    def __init__(self, device):
        self.device = device

    def __enter__(self):
        self.found = _Generators(self.device).states

    def __exit__(self, error, *_):
        if error is None and not all(map(torch.equal, self.found, _Generators(self.device).states)):
            raise RuntimeError("PolicyTrunk.backward: a block draws random numbers, and its forward pass was captured into a CUDA "
                               "graph, which kept no generator's state to draw them again")


@dataclass
class BlockNorms:
    """The vectors [d] around one block: the norm in front of it, and behind it a norm (gamma_post may be None) and a gate
    (None for none) of what it adds to the residual stream.  A gate may also have a value for every element of a batch, [T, d] in
    the embedding's type; its gradient has that shape and type then."""
    gamma_pre: torch.Tensor
    beta_pre: Any = None
    gamma_post: Any = None
    beta_post: Any = None
    gate: Any = None


class PolicyTrunk:
    """embedding [vocab, d]; blocks: callables; norms: a BlockNorms for each.  forward(token_ids, mask) gives x [T, d], the
    residual stream after the last block (padding tokens: mask 0, zero rows), and keeps what backward(dx) needs; with
    save=False (a decoding step, say) it keeps nothing.  backward gives a dict: "embedding" (or, with dhead, the tied head's
    gradient, to which it is added), "norms" (a dict for each block) and "blocks" (for each block the gradients of the
    tensors in `params[l]`, in order, None where its output does not depend on one)."""

    def __init__(self, embedding, blocks, norms, params=None, *, kind=TURNOPD_RMS_NORM, eps=1e-6, scale=1.0, resid_scale=1.0,
                 branch_scale=1.0, resid_dtype=None, keep=None):
        if len(blocks) != len(norms) or not blocks:
            raise ValueError("a BlockNorms for each block, and one block at least")
        if keep is not None and keep not in CODES:
            raise ValueError("keep must be None, 'e4m3' or 'int8'")
        self.embedding, self.blocks, self.norms = embedding, list(blocks), list(norms)
        self.params = list(params) if params is not None else [[] for _ in blocks]
        self.kind, self.eps, self.scale = int(kind), float(eps), float(scale)
        self.resid_scale, self.branch_scale, self.keep = float(resid_scale), float(branch_scale), keep
        self.resid_dtype = resid_dtype or embedding.dtype
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=embedding.device)
        self.saved = None

    def _put_away(self, x):
        if self.keep is None:
            return x
        codes = torch.empty(x.shape, dtype=CODES[self.keep], device=x.device)
        exps = torch.empty((x.shape[0], (x.shape[1] + 31) // 32), dtype=torch.uint8, device=x.device)
        turnopd_act8_store(x, self.mask, codes, exps, self.dev_status)
        return codes, exps

    def _take_back(self, kept, dtype):
        if self.keep is None:
            return kept
        out = torch.empty(kept[0].shape, dtype=dtype, device=kept[0].device)
        turnopd_act8_load(*kept, out)
        return out

    @torch.no_grad()
    def forward(self, token_ids, mask=None, save=True):
        self.token_ids, self.mask, self.saved = token_ids, mask, None
        T, d, dev, bt = token_ids.numel(), self.embedding.shape[1], self.embedding.device, self.embedding.dtype
        f32 = dict(dtype=torch.float32, device=dev)
        r = torch.empty((T, d), dtype=self.resid_dtype, device=dev)
        turnopd_embedding_fwd(self.embedding, token_ids, mask, self.scale, r, self.dev_status)
        h, stats = torch.empty((T, d), dtype=bt, device=dev), torch.zeros((T, 4), **f32)
        mean, rstd = torch.empty(T, **f32), torch.empty(T, **f32)
        n = self.norms[0]
        turnopd_norm_fwd(r, n.gamma_pre, n.beta_pre, mask, self.kind, self.eps, h, mean, rstd, self.dev_status)
        stats[:, 2], stats[:, 3] = mean, rstd
        autocast = _Autocast()
        saved = [dict(autocast=autocast, r=self._put_away(r), stats=stats)] if save else None
        for k, block in enumerate(self.blocks):
            n, after = self.norms[k], self.norms[k + 1] if k + 1 < len(self.blocks) else None
            if save:
                drawn = _NoDraws(dev) if torch.cuda.is_current_stream_capturing() else _Generators(dev)
            with autocast():
                y = block(h)
            r_next, stats = torch.empty_like(r), torch.empty((T, 4), **f32)
            h_next = torch.empty_like(h) if after else None
            turnopd_block_norm_fwd(r, y, n.gamma_post, n.beta_post, n.gate, after.gamma_pre if after else None,
                                   after.beta_pre if after else None, mask, self.kind, self.eps, self.resid_scale,
                                   self.branch_scale, r_next, h_next, stats, self.dev_status)
            if save:
                needs_y = n.gamma_post is not None or n.gate is not None
                saved.append(dict(h=self._put_away(h), y=self._put_away(y) if needs_y else None,
                                  r=self._put_away(r_next) if after else None, stats=stats, drawn=drawn))
            r, h = r_next, h_next
        self.saved = saved
        return r

    def backward(self, dx, dhead=None):
        """dx [T, d], of the residual stream's type: dL/dx.  It is used up; once after each forward pass that was saved."""
        if self.saved is None:
            raise RuntimeError("PolicyTrunk.backward needs a saved forward pass of its own")
        if torch.cuda.is_current_stream_capturing():
            raise RuntimeError("PolicyTrunk.backward cannot be captured: autograd runs the blocks, whose parameters may have "
                               "other graphs' nodes")
        saved, self.saved = self.saved, None
        T, d, dev, bt = dx.shape[0], dx.shape[1], dx.device, self.embedding.dtype
        f32 = dict(dtype=torch.float32, device=dev)
        ws = torch.empty(max(turnopd_block_norm_bwd_workspace_bytes(T, d), 256), dtype=torch.uint8, device=dev)
        norm_grads, block_grads = [dict() for _ in self.blocks], [None] * len(self.blocks)
        vector = lambda like: torch.empty(d, **f32) if like is not None else None  # noqa: E731
        dr, dh = dx, None
        for k in reversed(range(len(self.blocks))):
            n, s, after = self.norms[k], saved[k + 1], self.norms[k + 1] if dh is not None else None
            dy = torch.empty((T, d), dtype=bt, device=dev)
            gate = torch.empty((T, d), dtype=bt, device=dev) if n.gate is not None and n.gate.dim() == 2 else vector(n.gate)
            g = dict(gate=gate, gamma_post=vector(n.gamma_post), beta_post=vector(n.beta_post))
            pre = dict(gamma_pre=vector(after.gamma_pre), beta_pre=vector(after.beta_pre)) if after else dict(gamma_pre=None, beta_pre=None)
            with torch.no_grad():
                turnopd_block_norm_bwd(s["r"], s["y"], n.gamma_post, n.beta_post, n.gate, after.gamma_pre if after else None,
                                       self.mask, self.kind, self.resid_scale, self.branch_scale, s["stats"], dh, dr, dr, dy,
                                       g["gate"], g["gamma_post"], g["beta_post"], pre["gamma_pre"], pre["beta_pre"], ws)
            norm_grads[k].update(g)
            if after:
                norm_grads[k + 1].update(pre)
            h = self._take_back(s["h"], bt).detach().requires_grad_()
            with torch.enable_grad(), s["drawn"], saved[0]["autocast"]():
                y = self.blocks[k](h)
            leaves = [h, *self.params[k]]
            dh, *block_grads[k] = (torch.autograd.grad(y, leaves, dy, allow_unused=True) if y.requires_grad
                                   else [None] * len(leaves))  # its output depends on none of them
            dh = torch.zeros_like(h) if dh is None else dh.contiguous()
            saved[k + 1] = None
        n, s = self.norms[0], saved[0]
        norm_grads[0].update(gamma_pre=vector(n.gamma_pre), beta_pre=vector(n.beta_pre))
        with torch.no_grad():
            turnopd_block_norm_bwd(s["r"], None, None, None, None, n.gamma_pre, self.mask, self.kind, 1.0, 1.0, s["stats"], dh, dr,
                                   dr, None, None, None, None, norm_grads[0]["gamma_pre"], norm_grads[0]["beta_pre"], ws)
            V = self.embedding.shape[0]
            wse = torch.empty(turnopd_embedding_bwd_workspace_bytes(T, d, V), dtype=torch.uint8, device=dev)
            out = torch.empty((V, d), dtype=self.embedding.dtype, device=dev) if dhead is None else dhead
            turnopd_embedding_bwd(dr, self.token_ids, self.mask, self.scale, out, 0 if dhead is None else TURNOPD_ACCUMULATE_GRAD,
                                  wse, self.dev_status)
        return dict(embedding=out, norms=norm_grads, blocks=block_grads)

    def status(self) -> int:
        return int(self.dev_status.item())
