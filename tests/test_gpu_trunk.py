"""The model around its blocks as one chain -- embedding, blocks with their norms, gates and residual connections, policy head
with a tied table, and back -- against float64 autograd of the same model.

Tolerances, in the 2-norm.  fp32 throughout: a chain of some thirty roundings of 2^-24 and sums good to 1e-5: 1e-3.  bf16:
each activation and gradient on the way is rounded to 2^-8 at most, about 2^-9 in the mean square, some ten times in
sequence: 4 %.  8-bit activations change no value of the forward pass; each kept one is off by 2^-4 of itself at most
(e4m3; 2.6 % in the mean square), or 1.1 % of its group (int8, in the mean square for normals), and a gradient goes through
four of them in each of two blocks: 25 % and 10 %.
"""
import pytest
import torch

import paper_2607_05804_gb300 as P
import workloads as W
from paper_2607_05804_gb300.policy import PolicyHead
from paper_2607_05804_gb300.trunk import BlockNorms, PolicyTrunk

pytestmark = pytest.mark.gpu
LAYER, RMS = P.TURNOPD_LAYER_NORM, P.TURNOPD_RMS_NORM


def relative(a, b):
    return float((a.double() - b.double()).norm() / b.double().norm())


class Block:
    """Tokens mixed with the one before them, and a small network."""

    def __init__(self, w1, w2):
        self.w1, self.w2 = w1, w2

    def __call__(self, h):
        h = h + 0.5 * torch.cat([torch.zeros_like(h[:1]), h[:-1]])
        return torch.tanh(h @ self.w1) @ self.w2


def norm64(x, gamma, beta, kind, eps):
    mu = x.mean(1, keepdim=True) if kind == LAYER else 0.0
    h = (x - mu) / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps) * gamma
    return h + beta if beta is not None else h


def make(kind, d, V, dtype, seed=0):
    b = W.packed(seed=seed, num_traj=3, traj_len=200)
    g = torch.Generator(device="cuda").manual_seed(seed)
    rand = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    T = b.num_tokens
    leaf = lambda t: t.to(dtype).requires_grad_()  # noqa: E731
    table = leaf(rand(V, d) / d ** 0.5)
    ids = (V ** torch.rand(T, generator=g, device="cuda")).long().clamp(1, V).sub(1).int()
    blocks, norms, params = [], [], []
    for k in range(2):
        w1, w2 = leaf(rand(d, 96) / d ** 0.5), leaf(rand(96, d) / 96 ** 0.5)
        blocks.append(Block(w1, w2))
        params.append([w1, w2])
        beta = lambda: leaf(0.1 * rand(d)) if kind == LAYER else None  # noqa: E731
        norms.append(BlockNorms(leaf(1 + 0.2 * rand(d)), beta(), *((leaf(1 + 0.2 * rand(d)), beta()) if k == 0 else (None, None)),
                                gate=leaf(0.5 + 0.2 * rand(d)) if k == 0 else None))
    final = (leaf(1 + 0.2 * rand(d)), leaf(0.1 * rand(d)) if kind == LAYER else None)
    return b, T, table, ids, blocks, norms, params, final, rand


VECTORS = ("gamma_pre", "beta_pre", "gamma_post", "beta_post", "gate")


@pytest.mark.parametrize("kind,d", [(RMS, 256), (LAYER, 200), (RMS, 1001)])
@pytest.mark.parametrize("dtype,keep,tol", [(torch.float32, None, 1e-3), (torch.bfloat16, None, 0.04), (torch.float32, "e4m3", 0.25),
                                            (torch.float32, "int8", 0.1)])
def test_model_and_its_gradients(kind, d, dtype, keep, tol):
    V, scale, alpha, s = 700, d ** 0.5, 0.9, 0.5
    b, T, table, ids, blocks, norms, params, final, rand = make(kind, d, V, dtype)
    mask = torch.from_numpy(b.loss_mask).cuda()
    trunk = PolicyTrunk(table, blocks, norms, params, kind=kind, scale=scale, resid_scale=alpha, branch_scale=s, keep=keep)
    y = torch.randint(V, (T,), device="cuda").int()
    head = PolicyHead(final[0], table, mask, y, beta=final[1], kind=kind)
    x = trunk.forward(ids)
    lp, H = head.forward(x)
    gl, gh = rand(T), 0.1 * rand(T)
    dx, dgamma, dbeta, dhead = head.backward(gl, gh)
    own_head = dhead.clone()
    out = trunk.backward(dx, dhead=dhead)
    assert trunk.status() == 0 and head.status() == 0 and out["embedding"] is dhead

    leaves = {}
    wide = lambda t: leaves.setdefault(id(t), t.detach().double().requires_grad_()) if t is not None else None  # noqa: E731
    t64 = wide(table)
    r = t64[ids.long()] * scale
    for blk, n in zip(blocks, norms):
        h = norm64(r, wide(n.gamma_pre), wide(n.beta_pre), kind, 1e-6)
        v = Block(wide(blk.w1), wide(blk.w2))(h)
        if n.gamma_post is not None:
            v = norm64(v, wide(n.gamma_post), wide(n.beta_post), kind, 1e-6)
        r = alpha * r + s * (wide(n.gate) * v if n.gate is not None else v)
    assert relative(x, r.detach()) < (0.02 if dtype is torch.bfloat16 else 1e-4)
    ls = torch.log_softmax(norm64(r, wide(final[0]), wide(final[1]), kind, 1e-6) @ t64.T, 1)
    on = mask.bool()
    lp64, H64 = ls.gather(1, y[:, None].long())[:, 0], -(ls.exp() * ls).sum(1)
    loss = (gl.double()[on] * lp64[on]).sum() + (gh.double()[on] * H64[on]).sum()
    loss.backward()
    # the tied table has both gradients; what came through the embedding is the difference
    assert relative(out["embedding"], t64.grad) < tol
    assert float((out["embedding"].double() - own_head.double()).norm()) > 0
    for k, n in enumerate(norms):
        for name in VECTORS:
            p = getattr(n, name)
            if p is not None:
                assert relative(out["norms"][k][name], leaves[id(p)].grad) < tol, (k, name)
        for got, p in zip(out["blocks"][k], params[k]):
            assert relative(got, leaves[id(p)].grad) < tol
    with pytest.raises(RuntimeError):
        trunk.backward(dx)


def test_padding_and_an_untied_table():
    """Padding tokens give zero rows on the way and add nothing to any gradient; without a head's gradient the table's is whole."""
    kind, d, V = RMS, 256, 700
    b, T, table, ids, blocks, norms, params, _, rand = make(kind, d, V, torch.float32)
    blocks = [lambda h, blk=blk: torch.tanh(h @ blk.w1) @ blk.w2 for blk in blocks]  # each token by itself
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[T // 2:] = 0
    g = rand(T, d)
    outs = []
    for n, m in ((T, mask), (T // 2, None)):
        trunk = PolicyTrunk(table, blocks, norms, params, kind=kind, scale=2.0, resid_dtype=torch.float32)
        x = trunk.forward(ids[:n].contiguous(), m)
        assert not x[T // 2:].any()
        out = trunk.backward(g[:n].clone())
        assert trunk.status() == 0
        outs.append((x[:T // 2], out))
    (xa, a), (xb, c) = outs
    assert relative(xa, xb) < 1e-6 and relative(a["embedding"], c["embedding"]) < 1e-5
    seen = torch.zeros(V, dtype=torch.bool, device="cuda")
    seen[ids[:T // 2].long()] = True
    assert not a["embedding"][~seen].any()
    for k in range(2):
        for name in a["norms"][k]:
            if a["norms"][k][name] is not None:
                assert relative(a["norms"][k][name], c["norms"][k][name]) < 1e-5


def test_single_token():
    """A decoding step keeps nothing and gives the row that the whole batch gives."""
    kind, d, V = RMS, 256, 700
    b, T, table, ids, blocks, norms, params, _, _ = make(kind, d, V, torch.bfloat16)
    blocks = [lambda h, blk=blk: torch.tanh(h @ blk.w1) @ blk.w2 for blk in blocks]
    trunk = PolicyTrunk(table, blocks, norms, params, kind=kind)
    whole = trunk.forward(ids)
    one = trunk.forward(ids[7:8].contiguous(), save=False)
    assert relative(one, whole[7:8]) < 0.02 and trunk.status() == 0  # its blocks' products are summed in another order
    with pytest.raises(RuntimeError):
        trunk.backward(one)


def test_what_does_not_fit():
    t = torch.zeros((4, 8), device="cuda")
    with pytest.raises(ValueError):
        PolicyTrunk(t, [], [])
    with pytest.raises(ValueError):
        PolicyTrunk(t, [lambda h: h], [BlockNorms(t[0])], keep="fp4")


class Drawing:
    """A block that draws from torch's generators, on the device and on the host, or has its draws given."""

    def __init__(self, block, given=None):
        self.w1, self.w2, self.given, self.drawn = block.w1, block.w2, given, []

    def __call__(self, h):
        m, a = self.given if self.given else (2.0 * (torch.rand(h.shape, device=h.device) < 0.5), torch.rand(()))
        self.drawn.append((m, a))
        return torch.tanh((h * m) @ self.w1) @ self.w2 * float(a)


def test_blocks_that_draw_random_numbers():
    """The backward pass draws what the forward pass drew, whatever was drawn in between, and leaves the generators alone.  The
    same kernels run on the same numbers as with the draws given, up to the order of a product's sums."""
    kind, d, V = RMS, 200, 300
    b, T, table, ids, blocks, norms, params, _, rand = make(kind, d, V, torch.float32)
    drawing = [Drawing(blk) for blk in blocks]
    g = rand(T, d)
    trunk = PolicyTrunk(table, drawing, norms, params, kind=kind)
    x = trunk.forward(ids)
    torch.rand(7, device="cuda"), torch.rand(3)
    states = torch.get_rng_state(), torch.cuda.get_rng_state()
    out = trunk.backward(g.clone())
    assert torch.equal(torch.get_rng_state(), states[0]) and torch.equal(torch.cuda.get_rng_state(), states[1])
    for blk in drawing:
        (m, a), (m2, a2) = blk.drawn
        assert torch.equal(m, m2) and torch.equal(a, a2)
    assert not torch.equal(drawing[0].drawn[0][0], drawing[1].drawn[0][0])
    fixed = PolicyTrunk(table, [Drawing(blk, blk.drawn[0]) for blk in drawing], norms, params, kind=kind)
    assert relative(fixed.forward(ids), x) < 1e-5
    want = fixed.backward(g.clone())
    assert relative(out["embedding"], want["embedding"]) < 1e-5
    for k in range(2):
        assert relative(out["norms"][k]["gamma_pre"], want["norms"][k]["gamma_pre"]) < 1e-5
        assert all(relative(p, q) < 1e-5 for p, q in zip(out["blocks"][k], want["blocks"][k]))
    # a forward pass that keeps nothing draws what it draws without the trunk
    torch.manual_seed(5)
    trunk.forward(ids, save=False)
    torch.manual_seed(5)
    assert torch.equal(drawing[0].drawn[-1][0], 2.0 * (torch.rand((T, d), device="cuda") < 0.5))


def test_backward_of_a_captured_forward_pass():
    """Blocks that repeat themselves are taken back through from the values of the last replay; blocks that draw are refused."""
    kind, d, V = RMS, 200, 300
    b, T, table, ids, blocks, norms, params, _, rand = make(kind, d, V, torch.float32)
    g = rand(T, d)
    for own, draws in ((blocks, False), ([Drawing(blk) for blk in blocks], True)):
        trunk = PolicyTrunk(table, own, norms, params, kind=kind)
        trunk.forward(ids, save=False)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            x = trunk.forward(ids)
        graph.replay()
        if draws:
            with pytest.raises(RuntimeError, match="draws random numbers"):
                trunk.backward(g.clone())
            continue
        out = trunk.backward(g.clone())
        eager = PolicyTrunk(table, own, norms, params, kind=kind)
        assert relative(x, eager.forward(ids)) < 1e-5
        want = eager.backward(g.clone())
        assert relative(out["embedding"], want["embedding"]) < 1e-5
        assert all(relative(p, q) < 1e-5 for k in range(2) for p, q in zip(out["blocks"][k], want["blocks"][k]))


@pytest.mark.parametrize("inside", [False, True])
def test_blocks_under_autocast(inside):
    """The backward pass runs a block as the forward pass ran it, called inside of the autocast context or outside of it."""
    kind, d, V = RMS, 200, 300
    b, T, table, ids, blocks, norms, params, _, rand = make(kind, d, V, torch.float32)
    seen = []

    def cast(blk):
        def run(h):
            y = torch.tanh(h @ blk.w1) @ blk.w2
            seen.append(y.dtype)
            return y.float()
        return run

    trunk = PolicyTrunk(table, [cast(blk) for blk in blocks], norms, params, kind=kind)
    g = rand(T, d)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        trunk.forward(ids)
        out = trunk.backward(g.clone()) if inside else None
    out = out or trunk.backward(g.clone())
    assert seen == [torch.bfloat16] * 4
    assert all(p is not None and p.dtype is torch.float32 and bool(p.any()) for k in range(2) for p in out["blocks"][k])
    # and the other way round
    seen.clear()
    trunk.forward(ids)
    with torch.autocast("cuda", dtype=torch.bfloat16):
        trunk.backward(g.clone())
        assert torch.is_autocast_enabled() and torch.is_autocast_cache_enabled()
    assert seen == [torch.float32] * 4


def test_a_block_whose_output_depends_on_nothing():
    """What comes back goes on through the residual stream alone; the parameters of such a block have no gradient."""
    kind, d, V = RMS, 200, 300
    b, T, table, ids, _, norms, params, _, rand = make(kind, d, V, torch.float32)
    dx = rand(T, d)
    trunk = PolicyTrunk(table, [torch.ones_like] * 2, norms, params, kind=kind, scale=2.0, resid_scale=0.5)
    trunk.forward(ids)
    out = trunk.backward(dx.clone())
    assert trunk.status() == 0 and out["blocks"] == [[None, None], [None, None]]
    want = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, ids.long(), dx.double()) * 0.5
    assert relative(out["embedding"], want) < 1e-5
    assert not out["norms"][0]["gamma_pre"].any() and out["norms"][0]["gate"].any()


@pytest.mark.parametrize("dtype,keep,tol", [(torch.float32, None, 1e-3), (torch.bfloat16, None, 0.04), (torch.float32, "int8", 0.1)])
def test_a_gate_for_every_element(dtype, keep, tol):
    """Gates [T, d], on a block with a norm behind it and on one without, with a mask: every gradient against autograd."""
    kind, d, V = RMS, 200, 300
    b, T, table, ids, blocks, norms, params, _, rand = make(kind, d, V, dtype)
    mask = torch.from_numpy(b.loss_mask).cuda()
    on = mask.bool()
    for n in norms:
        n.gate = torch.sigmoid(rand(T, d)).to(dtype).requires_grad_()
    norms[0].beta_post = (0.2 * rand(d)).to(dtype).requires_grad_()
    blocks = [lambda h, blk=blk: torch.tanh(h @ blk.w1) @ blk.w2 for blk in blocks]  # each token by itself
    trunk = PolicyTrunk(table, blocks, norms, params, kind=kind, branch_scale=0.5, keep=keep)
    x = trunk.forward(ids, mask)
    g = rand(T, d).to(dtype)
    g64 = g.double()[on]
    out = trunk.backward(g)
    assert trunk.status() == 0
    leaves = {}
    wide = lambda t: leaves.setdefault(id(t), t.detach().double().requires_grad_()) if t is not None else None  # noqa: E731
    r = wide(table)[ids.long()][on]
    for (w1, w2), n in zip(params, norms):
        v = torch.tanh(norm64(r, wide(n.gamma_pre), None, kind, 1e-6) @ wide(w1)) @ wide(w2)
        if n.gamma_post is not None:
            v = norm64(v, wide(n.gamma_post), wide(n.beta_post), kind, 1e-6)
        r = r + 0.5 * wide(n.gate)[on] * v
    assert relative(x[on], r.detach()) < (0.02 if dtype is torch.bfloat16 else 1e-4)
    (g64 * r).sum().backward()
    assert relative(out["embedding"], leaves[id(table)].grad) < tol
    for k, n in enumerate(norms):
        assert out["norms"][k]["gate"].shape == (T, d) and not out["norms"][k]["gate"][~on].any()
        for name in VECTORS:
            if getattr(n, name) is not None:
                assert relative(out["norms"][k][name], leaves[id(getattr(n, name))].grad) < tol, (k, name)
        for got, p in zip(out["blocks"][k], params[k]):
            assert relative(got, leaves[id(p)].grad) < tol


def test_decoding_step_in_a_graph():
    """A step captured once gives the hidden states of whatever tokens its buffer holds; products of the same sizes, fp32."""
    kind, d, V = RMS, 256, 700
    b, T, table, ids, blocks, norms, params, _, _ = make(kind, d, V, torch.float32)
    trunk = PolicyTrunk(table, blocks, norms, params, kind=kind)
    step = ids[:4].clone()
    trunk.forward(step, save=False)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        x = trunk.forward(step, save=False)
    for k in (4, 100, 200):
        step.copy_(ids[k:k + 4])
        graph.replay()
        assert relative(x, PolicyTrunk(table, blocks, norms, params, kind=kind).forward(step, save=False)) < 1e-5
    assert trunk.status() == 0
