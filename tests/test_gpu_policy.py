"""The policy head as one chain -- norm, LM head, log probabilities, and the gradients back -- against float64 autograd,
and the norm in front of the fused LM head.

Tolerance of the chain: bf16 hidden states, logits, dlogits and dh are each rounded to 2^-9 of themselves; a logit of up to 8
is off by up to 2^-6, and p by as much: gradients agree to 2 % in the 2-norm, 4 % allowed.
"""
import pytest
import torch

import paper_2607_05804_gb300 as P
import workloads as W
from paper_2607_05804_gb300.policy import PolicyHead

pytestmark = pytest.mark.gpu


def relative(a, b):
    return float((a.double() - b).norm() / b.norm())


def setup(kind, d, V, seed=0):
    b = W.packed(seed=seed, num_traj=3, traj_len=300)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    T = b.num_tokens
    x = (rand(T, d) * 2 + 0.3).bfloat16()
    gamma, beta = (1 + 0.2 * rand(d)).bfloat16(), (0.1 * rand(d)).bfloat16() if kind == P.TURNOPD_LAYER_NORM else None
    head = (rand(V, d) * 1.5 / d ** 0.5).bfloat16()
    mask = torch.from_numpy(b.loss_mask).cuda()
    y = torch.randint(V, (T,), generator=g, device="cuda").int()
    return b, x, gamma, beta, head, mask, y, rand


def norm64(x, gamma, beta, kind, eps):
    mu = x.mean(1, keepdim=True) if kind == P.TURNOPD_LAYER_NORM else 0.0
    h = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps) * gamma
    return h + beta if beta is not None else h


@pytest.mark.parametrize("kind,d,V", [(P.TURNOPD_RMS_NORM, 512, 3001), (P.TURNOPD_LAYER_NORM, 264, 1000)])
def test_policy_head(kind, d, V):
    b, x, gamma, beta, head, mask, y, rand = setup(kind, d, V)
    ph = PolicyHead(gamma, head, mask, y, beta=beta, kind=kind, n_top=5)
    lp, H = ph.forward(x)
    at = mask.nonzero()[:, 0]
    gl, gh = rand(mask.numel()), 0.1 * rand(mask.numel())
    leaves = [t.double().requires_grad_() for t in (x, gamma, head)] + ([beta.double().requires_grad_()] if beta is not None else [])
    h64 = norm64(leaves[0], leaves[1], leaves[3] if beta is not None else None, kind, 1e-6)
    ls = torch.log_softmax(h64[at] @ leaves[2].T, 1)
    lp64, H64 = ls.gather(1, y[at, None].long())[:, 0], -(ls.exp() * ls).sum(1)
    assert relative(lp[at], lp64.detach()) < 0.01 and relative(H[at], H64.detach()) < 0.01
    assert not lp[mask == 0].any() and not H[mask == 0].any()
    best = torch.sort(ph.logits.double(), dim=1, descending=True, stable=True).indices[:, :5]
    assert torch.equal(ph.top_ids[at].long(), best)
    grads = torch.autograd.grad((gl.double()[at] * lp64).sum() + (gh.double()[at] * H64).sum(), leaves)
    dx, dgamma, dbeta, dhead = ph.backward(gl, gh)
    assert ph.status() == 0 and not dx[mask == 0].any()
    assert relative(dx, grads[0]) < 0.04 and relative(dgamma, grads[1]) < 0.04 and relative(dhead, grads[2]) < 0.04
    if beta is not None:
        assert relative(dbeta, grads[3]) < 0.04
    # mean entropy by turn index
    tid, off = torch.from_numpy(b.turn_id).cuda(), torch.from_numpy(b.traj_offsets).cuda()
    got = ph.turn_entropy(tid, off, b.max_turns)
    for t in range(b.max_turns):
        on = (tid == t) & (mask == 1)
        want = H[on].double().mean() if bool(on.any()) else torch.zeros((), device="cuda", dtype=torch.float64)
        assert abs(got[t] - want) <= 1e-9 + 1e-9 * want


def test_batch_without_a_supervised_token():
    """All zeros, as a rank of a data-parallel step may meet it."""
    b, x, gamma, beta, head, mask, y, rand = setup(P.TURNOPD_LAYER_NORM, 264, 1000)
    mask = torch.zeros_like(mask)
    ph = PolicyHead(gamma, head, mask, y, beta=beta, kind=P.TURNOPD_LAYER_NORM, n_top=5)
    lp, H = ph.forward(x)
    assert not lp.any() and not H.any() and (ph.top_ids == -1).all() and not ph.top_logprob.any()
    grads = ph.backward(rand(mask.numel()), rand(mask.numel()))
    for got, shape in zip(grads, (x.shape, gamma.shape, beta.shape, head.shape)):
        assert got.shape == shape and not got.any()
    tid, off = torch.from_numpy(b.turn_id).cuda(), torch.from_numpy(b.traj_offsets).cuda()
    assert not ph.turn_entropy(tid, off, b.max_turns).any()
    assert ph.status() == 0


def test_parameters_that_require_gradients():
    """A model's own parameters and hidden states: the same numbers, and nothing recorded for autograd."""
    b, x, gamma, beta, head, mask, y, rand = setup(P.TURNOPD_LAYER_NORM, 264, 1000)
    gl, gh = rand(mask.numel()), rand(mask.numel())
    outs = []
    for wrap in (lambda t: t, lambda t: torch.nn.Parameter(t.clone())):
        ph = PolicyHead(wrap(gamma), wrap(head), mask, y, beta=wrap(beta), kind=P.TURNOPD_LAYER_NORM)
        xx = wrap(x)
        lp, H = ph.forward(xx)
        out = [t.clone() for t in (lp, H)] + [t.clone() for t in ph.backward(gl, gh)]
        assert ph.status() == 0 and not any(t.requires_grad for t in out)
        outs.append(out)
    assert all(torch.equal(a, b) for a, b in zip(*outs))


def test_a_backward_pass_to_each_forward_pass():
    """The logits hold their gradient after a backward pass: a second one has nothing to start from and is refused."""
    b, x, gamma, beta, head, mask, y, rand = setup(P.TURNOPD_RMS_NORM, 256, 1000)
    ph = PolicyHead(gamma, head, mask, y)
    gl = rand(mask.numel())
    with pytest.raises(RuntimeError):
        ph.backward(gl)
    ph.forward(x)
    first = [t.clone() for t in ph.backward(gl) if t is not None]
    with pytest.raises(RuntimeError):
        ph.backward(gl)
    ph.forward(x)
    again = [t for t in ph.backward(gl) if t is not None]
    assert ph.status() == 0 and all(torch.equal(a, b) for a, b in zip(first, again))


def test_norm_in_front_of_the_fused_head():
    """The distillation step from the last block's output: norm, both LM heads in the loss, and back through the norm."""
    d, d_t, V = 256, 320, 2000
    b, x, gamma, _, head, mask, _, rand = setup(P.TURNOPD_RMS_NORM, d, V)
    T = mask.numel()
    h_t, W_t = rand(T, d_t).bfloat16(), (rand(V, d_t) * 1.5 / d_t ** 0.5).bfloat16()
    w = torch.rand(T, device="cuda") / T * mask
    h, rstd = torch.empty_like(x), torch.empty(T, device="cuda")
    dh, dx = torch.empty((T, d), device="cuda"), torch.empty_like(x)
    token_loss, loss = torch.empty(T, device="cuda"), torch.zeros(1, dtype=torch.float64, device="cuda")
    dgamma, st = torch.empty(d, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.turnopd_fused_workspace_bytes(T, V, d, d_t), dtype=torch.uint8, device="cuda")
    ws_n = torch.empty(P.turnopd_norm_bwd_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")
    P.turnopd_norm_fwd(x, gamma, None, mask, P.TURNOPD_RMS_NORM, 1e-6, h, None, rstd, st)
    P.turnopd_fused_lmhead_fwd_bwd(h, head, h_t, W_t, mask, w, P.TURNOPD_FULL_VOCAB, dh, token_loss, loss, ws, st)
    P.turnopd_norm_bwd(x, gamma, mask, P.TURNOPD_RMS_NORM, None, rstd, dh, dx, dgamma, None, ws_n)
    assert st.item() == 0
    x64, g64 = x.double().requires_grad_(), gamma.double().requires_grad_()
    ls = torch.log_softmax(norm64(x64, g64, None, P.TURNOPD_RMS_NORM, 1e-6) @ head.double().T, 1)
    lt = torch.log_softmax(h_t.double() @ W_t.double().T, 1)
    want = (w.double() * (ls.exp() * (ls - lt)).sum(1)).sum()
    gx, gg = torch.autograd.grad(want, (x64, g64))
    assert abs(loss.item() - want.item()) < 0.02 * abs(want.item())
    assert relative(dx, gx) < 0.04 and relative(dgamma, gg) < 0.04 and not dx[mask == 0].any()
