"""Performance cases of the operators around the loss: log probabilities of given tokens (with entropy and top
alternatives) and their gradient, and the final norm before the LM head with its backward pass.

A case is a plain dict.  ``op`` is "logprobs", "logprobs_bwd", "norm" or "norm_bwd"; common keys:

``tokens``  tokens of the packed batch; ``share`` of them are supervised, in runs as turns have them (1: no loss mask)
``vocab``, ``ld``, ``layout``  columns, row stride, and one row per token ("dense") or per supervised token ("compact")
``d``, ``pad``  columns of a hidden state, and elements between the end of one row and the start of the next

The number of supervised tokens follows from the case alone; the seed draws every value and where the runs lie.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

V_MAIN = 151_936
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}


def listed():
    """Twelve cases: one decoding step, ordinary batches of each operator, type and layout, and the largest."""
    return [
        # one decoding step of one rollout: the sampled token's log probability and five alternatives; latency is all
        dict(name="decode_1", op="logprobs", tokens=1, share=1.0, vocab=V_MAIN, ld=V_MAIN, layout="dense", logits="bf16",
             top=5, holes=0.0),
        # a decoding step of 64 rollouts, fp32 logits, a grammar that forbids nine tenths of the vocabulary
        dict(name="decode_64_grammar_f32", op="logprobs", tokens=64, share=1.0, vocab=V_MAIN, ld=V_MAIN, layout="dense",
             logits="f32", top=20, holes=0.9),
        # scoring a packed batch of 8 trajectories before the update: log probabilities and entropies of what was sampled
        dict(name="score_packed", op="logprobs", tokens=16_384, share=0.6, vocab=V_MAIN, ld=V_MAIN, layout="compact",
             logits="bf16", top=0, holes=0.0),
        # scoring with alternatives where nobody padded the vocabulary: an odd row stride, one row per token
        dict(name="score_odd_top10", op="logprobs", tokens=4096, share=0.6, vocab=50_001, ld=50_001, layout="dense",
             logits="bf16", top=10, holes=0.0),
        # the gradient of a policy term with an entropy bonus on a packed batch
        dict(name="policy_packed", op="logprobs_bwd", tokens=8192, share=0.6, vocab=V_MAIN, ld=V_MAIN, layout="compact",
             logits="bf16", grad="bf16", entropy=True, zero_masked=False),
        # the same without the bonus, fp32 rows of an odd stride, masked rows zeroed as autograd wants it
        dict(name="policy_odd_f32", op="logprobs_bwd", tokens=4096, share=0.6, vocab=50_001, ld=50_001, layout="dense",
             logits="f32", grad="f32", entropy=False, zero_masked=True),
        # a debugging batch of two short trajectories: launches are all it costs
        dict(name="policy_tiny_f32", op="logprobs_bwd", tokens=256, share=0.5, vocab=1024, ld=1024, layout="dense",
             logits="f32", grad="f32", entropy=True, zero_masked=True),
        # one token's final norm in a decoding step
        dict(name="norm_decode_1", op="norm", tokens=1, share=1.0, d=4096, pad=0, x="bf16", y="bf16", params="bf16",
             kind="rms", beta=False, stats=False),
        # the final norm of a packed batch; only supervised tokens go on to the head
        dict(name="norm_packed_rms", op="norm", tokens=32_768, share=0.6, d=4096, pad=0, x="bf16", y="bf16",
             params="bf16", kind="rms", beta=False, stats=True),
        # an odd width in fp32, every token wanted
        dict(name="norm_odd_layer_f32", op="norm", tokens=4096, share=1.0, d=1001, pad=0, x="f32", y="f32",
             params="f32", kind="layer", beta=True, stats=True),
        # its backward pass behind the fused LM head, which gives dL/dh in fp32 with zero rows for masked tokens
        dict(name="norm_bwd_packed", op="norm_bwd", tokens=32_768, share=0.6, d=5120, pad=0, x="bf16", dy="f32",
             dx="bf16", params="bf16", kind="layer", beta=True),
        # the same on one micro-batch
        dict(name="norm_bwd_micro_rms", op="norm_bwd", tokens=512, share=0.6, d=4096, pad=0, x="bf16", dy="f32",
             dx="bf16", params="bf16", kind="rms", beta=False),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("logprobs", "logprobs", "logprobs_bwd", "norm", "norm_bwd"))
    while True:
        share = rng.choice((1.0, round(rng.uniform(0.05, 0.95), 2)))
        if op in ("norm", "norm_bwd"):
            d = _log(rng, 128, 8192)
            d = d if rng.random() < 0.3 else max(64, d // 64 * 64)
            c = dict(op=op, tokens=_log(rng, 1, 32_768), share=share, d=d, pad=rng.choice((0, 0, 0, 8, 3)),
                     x=rng.choice(("bf16", "bf16", "f32")), params=rng.choice(("bf16", "f32")),
                     kind=rng.choice(("layer", "rms")))
            c["beta"] = c["kind"] == "layer" and rng.random() < 0.8
            if op == "norm":
                c.update(y=rng.choice(("bf16", c["x"])), stats=rng.random() < 0.7)
            else:
                c.update(dy=rng.choice(("f32", c["x"])), dx=c["x"])
        else:
            v = _log(rng, 1024, V_MAIN)
            v = v if rng.random() < 0.3 else v // 64 * 64
            c = dict(op=op, tokens=_log(rng, 1, 16_384), share=share, vocab=v,
                     ld=v if rng.random() < 0.7 else (v + 63) // 64 * 64, logits=rng.choice(("bf16", "bf16", "f32")))
            c["layout"] = rng.choice(("dense", "compact")) if share < 1.0 else "dense"
            if op == "logprobs":
                c.update(top=rng.choice((0, 0, 1, 5, 20, rng.randint(1, 32))), holes=rng.choice((0.0, 0.0, 0.5, 0.99)))
            else:
                c.update(grad=rng.choice((c["logits"], c["logits"], "f32")), entropy=rng.random() < 0.5,
                         zero_masked=share < 1.0 and c["layout"] == "dense" and rng.random() < 0.7)
        rows = c["tokens"] if c.get("layout") == "dense" else _supervised(c)
        if 3072 in c.values() or _supervised(c) < 1 or rows * c.get("vocab", 0) > 1_000_000_000:
            continue
        return c


# ---------------------------------------------------------------- inputs

def _supervised(case):
    return case["tokens"] if case["share"] >= 1.0 else int(round(case["share"] * case["tokens"]))


def _mask(case, seed):
    """Runs of observed and supervised tokens (as turns have them), the right number of the latter, turned by the seed."""
    T, n = case["tokens"], _supervised(case)
    rng = np.random.default_rng([T, n])
    m = np.zeros(T, np.uint8)
    runs = max(1, T // 200)
    cut = lambda total: np.diff(np.concatenate([[0], np.sort(rng.integers(0, total + 1, runs - 1)), [total]]))  # noqa: E731
    at = 0
    for off, on in zip(cut(T - n), cut(n)):
        m[at + off:at + off + on] = 1
        at += off + on
    return np.roll(m, int(np.random.default_rng(seed).integers(0, T)))


def _tokens(case, seed):
    """Loss mask, supervised tokens' indexes and the token -> row map, on the GPU."""
    T = case["tokens"]
    if case["share"] >= 1.0:
        return dict(mask=None, at=torch.arange(T, device="cuda"), rows=None)
    m = _mask(case, seed)
    at = np.nonzero(m)[0]
    rows = None
    if case.get("layout") == "compact":
        rows = np.full(T, -1, np.int32)
        rows[at] = np.arange(at.size, dtype=np.int32)
        rows = torch.from_numpy(rows).cuda()
    return dict(mask=torch.from_numpy(m).cuda(), at=torch.from_numpy(at).cuda(), rows=rows)


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _logits(case, n, seed):
    """n rows: normals of deviation 3, one id of each row raised by 0 to 30 (an unsure model, and one that is all but
    certain), a share of the vocabulary forbidden; and one token of each row drawn from its softmax."""
    gen, V, ld = _generator(seed), case["vocab"], case["ld"]
    z = torch.zeros((n, ld), dtype=TYPES[case["logits"]], device="cuda")
    y = torch.empty(n, dtype=torch.int32, device="cuda")
    step = max(1, 200_000_000 // V)
    for r in range(0, n, step):
        k = min(step, n - r)
        a = torch.randn((k, V), generator=gen, device="cuda").mul_(3.0)
        ids = torch.randint(V, (k, 1), generator=gen, device="cuda")
        if case.get("holes"):
            gone = torch.rand((1, V), generator=gen, device="cuda") < case["holes"]
            a.masked_fill_(gone, -math.inf)
        a.scatter_(1, ids, 30.0 * torch.rand((k, 1), generator=gen, device="cuda"))
        z[r:r + k, :V] = a
        e = torch.empty_like(a).exponential_(generator=gen).clamp_(min=1e-30)
        y[r:r + k] = torch.argmax(z[r:r + k, :V].float() - e.log_(), dim=1)
    return z, y


def _saved(z, y, V):
    """What the forward pass keeps for the backward pass: (m, log S), log p_y and H of each row."""
    out = []
    step = max(1, 50_000_000 // V)
    for r in range(0, z.shape[0], step):
        x = z[r:r + step, :V].double()
        m = x.amax(1, keepdim=True)
        x = x - m
        logs = x.exp().sum(1, keepdim=True).log()
        lp = x - logs
        py = lp.gather(1, y[r:r + step, None].long())
        out.append(torch.cat([m, logs, py, -(lp.exp() * lp).sum(1, keepdim=True)], 1))
    return torch.cat(out).float()


def prepare(case, seed):
    """What a program holds before the call: the inputs, and the buffers that the outputs go to."""
    s = dict(case=case, **_tokens(case, seed))
    T, at = case["tokens"], s["at"]
    f32 = dict(dtype=torch.float32, device="cuda")
    s["status"] = torch.zeros(1, dtype=torch.int32, device="cuda")
    if case["op"] in ("norm", "norm_bwd"):
        gen, d = _generator(seed), case["d"]
        put = lambda t: torch.zeros((T, d + case["pad"]), dtype=TYPES[t], device="cuda")[:, :d]  # noqa: E731
        # a residual stream: a few channels many times as large as the others, a mean that is not 0
        scale = torch.where(torch.rand(d, generator=gen, device="cuda") < 0.01, 30.0, 1.0)
        s["x"] = put(case["x"])
        s["x"].copy_(torch.randn((T, d), generator=gen, device="cuda") * scale + 0.3)
        s["gamma"] = (1.0 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(TYPES[case["params"]])
        s["beta"] = (0.1 * torch.randn(d, generator=gen, device="cuda")).to(TYPES[case["params"]]) if case["beta"] else None
        s["eps"] = 1e-6
        s["mean"], s["rstd"] = torch.zeros(T, **f32), torch.zeros(T, **f32)
        if case["op"] == "norm":
            s["y"] = put(case["y"])
            return s
        s["dy"] = put(case["dy"])
        s["dy"][at] = (1e-3 * torch.randn((at.numel(), d), generator=gen, device="cuda")).to(TYPES[case["dy"]])
        s["mean"][at], s["rstd"][at] = (v.float() for v in _moments64(s["x"][at].double(), case, s["eps"]))
        s["dx"] = put(case["dx"])
        s["dgamma"] = torch.zeros(d, **f32)
        s["dbeta"] = torch.zeros(d, **f32) if case["beta"] else None
        return s
    n = T if case["layout"] == "dense" else at.numel()
    s["logits"], y = _logits(case, n, seed)
    s["ids"] = torch.zeros(T, dtype=torch.int32, device="cuda")
    s["ids"][at] = y if n == at.numel() else y[at]
    if case["op"] == "logprobs":
        k = case["top"]
        s["logprob"], s["entropy"], s["stats"] = (torch.zeros(v, **f32) for v in (T, T, (T, 2)))
        s["top_ids"] = torch.zeros((T, k), dtype=torch.int32, device="cuda") if k else None
        s["top_logprob"] = torch.zeros((T, k), **f32) if k else None
        return s
    kept = torch.zeros((T, 4), **f32)
    kept[at] = _saved(s["logits"] if n == at.numel() else s["logits"][at], s["ids"][at], case["vocab"])
    s["stats"], s["logprob"], s["entropy"] = kept[:, :2].contiguous(), kept[:, 2].contiguous(), kept[:, 3].contiguous()
    gen = _generator(seed + 1)
    # advantages over the number of tokens; one weight of the entropy for all
    s["d_logprob"] = torch.randn(T, generator=gen, device="cuda") / at.numel()
    s["d_entropy"] = torch.full((T,), 0.01 / at.numel(), **f32) if case["entropy"] else None
    s["grad"] = torch.zeros(s["logits"].shape, dtype=TYPES[case["grad"]], device="cuda")
    return s


# ---------------------------------------------------------------- a pass

def run(s):
    return _own(s) if own else PLAIN[s["case"]["op"]](s)


def _own(s):
    import paper_2607_05804_gb300 as lib

    c = s["case"]
    if c["op"] == "logprobs":
        if "workspace" not in s:
            s["workspace"] = torch.empty(lib.turnopd_token_logprobs_workspace_bytes(c["tokens"]), dtype=torch.uint8, device="cuda")
        lib.turnopd_token_logprobs(s["logits"], c["vocab"], s["rows"], s["ids"], s["mask"], c["top"], s["logprob"],
                                   s["entropy"], s["stats"], s["top_ids"], s["top_logprob"], s["workspace"], s["status"])
        return {k: s[k] for k in ("logprob", "entropy", "stats", "top_ids", "top_logprob")}
    if c["op"] == "logprobs_bwd":
        if "workspace" not in s:
            s["workspace"] = torch.empty(lib.turnopd_token_logprobs_workspace_bytes(c["tokens"]), dtype=torch.uint8, device="cuda")
        lib.turnopd_token_logprobs_bwd(s["logits"], c["vocab"], s["rows"], s["ids"], s["mask"], s["stats"], s["logprob"],
                                       s["entropy"], s["d_logprob"], s["d_entropy"], s["grad"],
                                       lib.TURNOPD_ZERO_MASKED_GRAD if c["zero_masked"] else 0, s["workspace"], s["status"])
        return s["grad"]
    kind = lib.TURNOPD_RMS_NORM if c["kind"] == "rms" else lib.TURNOPD_LAYER_NORM
    if c["op"] == "norm":
        mean, rstd = (s["mean"] if c["kind"] == "layer" else None, s["rstd"]) if c["stats"] else (None, None)
        lib.turnopd_norm_fwd(s["x"], s["gamma"], s["beta"], s["mask"], kind, s["eps"], s["y"], mean, rstd, s["status"])
        return {"y": s["y"], "mean": mean, "rstd": rstd}
    if "workspace" not in s:
        s["workspace"] = torch.empty(lib.turnopd_norm_bwd_workspace_bytes(c["tokens"], c["d"]), dtype=torch.uint8, device="cuda")
    lib.turnopd_norm_bwd(s["x"], s["gamma"], s["mask"], kind, s["mean"] if c["kind"] == "layer" else None, s["rstd"], s["dy"],
                         s["dx"], s["dgamma"], s["dbeta"], s["workspace"])
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


def _supervised_rows(s):
    """The logits of the supervised tokens, one row each, in 32 bits."""
    z = s["logits"][:, :s["case"]["vocab"]]
    return (z[s["at"]] if z.shape[0] > s["at"].numel() else z).float()


def _plain_logprobs(s):
    c, at = s["case"], s["at"]
    z, y = _supervised_rows(s), s["ids"][at].long()[:, None]
    m = z.amax(1, keepdim=True)
    x = z - m
    p = x.exp()
    total = p.sum(1, keepdim=True)
    logs = total.log()
    s["stats"][at] = torch.cat([m, logs], 1)
    s["logprob"][at] = (x.gather(1, y) - logs)[:, 0]
    p.div_(total)
    s["entropy"][at] = logs[:, 0] - torch.where(p > 0, p.mul_(x), 0.0).sum(1)
    del p, x
    out = {k: s[k] for k in ("logprob", "entropy", "stats")}
    if c["top"]:
        # one 64-bit key for each logit: its value, then the lower id first
        key = (z + 0.0).view(torch.int32)
        key = torch.where(key < 0, key ^ 0x7fffffff, key).long() * 2**32 + (2**31 - 1 - torch.arange(z.shape[1], device="cuda"))
        best = (2**31 - 1) - (key.topk(c["top"], dim=1).values & 0xffffffff)
        s["top_ids"].fill_(-1)
        s["top_logprob"].zero_()
        s["top_ids"][at] = best.int()
        s["top_logprob"][at] = z.gather(1, best) - m - logs
        out.update(top_ids=s["top_ids"], top_logprob=s["top_logprob"])
    return out


def _plain_logprobs_bwd(s):
    c, at = s["case"], s["at"]
    lp = _supervised_rows(s)
    lp = lp.sub_(s["stats"][at, 0, None]).sub_(s["stats"][at, 1, None]) if c["logits"] == "bf16" else \
        lp - s["stats"][at, 0, None] - s["stats"][at, 1, None]
    p = lp.exp()
    gl = s["d_logprob"][at, None]
    g = p * -gl
    if s["d_entropy"] is not None:
        g -= s["d_entropy"][at, None] * p * (lp + s["entropy"][at, None])
    y = s["ids"][at].long()[:, None]
    g.scatter_add_(1, y, gl)
    dense = s["grad"].shape[0] > at.numel()
    if dense and c["zero_masked"]:
        s["grad"][:, :c["vocab"]].zero_()
    if dense:
        s["grad"][at, :c["vocab"]] = g.to(s["grad"].dtype)
    else:
        s["grad"][:, :c["vocab"]] = g
    return s["grad"]


def _plain_norm(s):
    c, at = s["case"], s["at"]
    x = (s["x"] if s["mask"] is None else s["x"][at]).float()
    mean = x.mean(1, keepdim=True) if c["kind"] == "layer" else 0.0
    x = x - mean
    rstd = (x.square().mean(1, keepdim=True) + s["eps"]).rsqrt()
    y = x * rstd * s["gamma"].float()
    if s["beta"] is not None:
        y += s["beta"].float()
    if s["mask"] is None:
        s["y"].copy_(y)
    else:
        s["y"].zero_()
        s["y"][at] = y.to(s["y"].dtype)
    out = {"y": s["y"], "mean": None, "rstd": None}
    if c["stats"]:
        s["rstd"][at] = rstd[:, 0]
        out["rstd"] = s["rstd"]
        if c["kind"] == "layer":
            s["mean"][at] = mean[:, 0]
            out["mean"] = s["mean"]
    return out


def _plain_norm_bwd(s):
    c, at = s["case"], s["at"]
    x, dy = (v.float() if s["mask"] is None else v[at].float() for v in (s["x"], s["dy"]))
    r = s["rstd"][at, None]
    xh = (x - s["mean"][at, None]) * r if c["kind"] == "layer" else x * r
    g = dy * s["gamma"].float()
    dx = g - xh * (g * xh).mean(1, keepdim=True)
    if c["kind"] == "layer":
        dx -= g.mean(1, keepdim=True)
    dx *= r
    if s["mask"] is None:
        s["dx"].copy_(dx)
    else:
        s["dx"].zero_()
        s["dx"][at] = dx.to(s["dx"].dtype)
    s["dgamma"].copy_((dy * xh).sum(0))
    if s["dbeta"] is not None:
        s["dbeta"].copy_(dy.sum(0))
    return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}


PLAIN = {"logprobs": _plain_logprobs, "logprobs_bwd": _plain_logprobs_bwd, "norm": _plain_norm, "norm_bwd": _plain_norm_bwd}


# ---------------------------------------------------------------- what a pass needs

def work(case):
    T, R = case["tokens"], _supervised(case)
    mask = T if case["share"] < 1.0 else 0
    if case["op"] in ("norm", "norm_bwd"):
        d, x = case["d"], BYTES[case["x"]]
        params = d * BYTES[case["params"]] * (2 if case["beta"] and case["op"] == "norm" else 1)
        kept = 8 if case["kind"] == "layer" else 4
        if case["op"] == "norm":
            return {"bytes": float(mask + R * d * x + T * d * BYTES[case["y"]] + params + (T * kept if case["stats"] else 0)),
                    "flops": 8.0 * R * d}
        return {"bytes": float(mask + R * (d * (x + BYTES[case["dy"]]) + kept) + T * d * BYTES[case["dx"]] + params
                               + 4 * d * (2 if case["beta"] else 1)), "flops": 12.0 * R * d}
    V, esz = case["vocab"], BYTES[case["logits"]]
    tokens = mask + R * (4 + (4 if case["layout"] == "compact" and mask else 0))
    if case["op"] == "logprobs":
        return {"bytes": float(tokens + R * V * esz + T * (16 + 8 * case["top"])), "flops": 5.0 * R * V}
    gsz = BYTES[case["grad"]]
    zeros = (T - R) * V * gsz if case["zero_masked"] else 0
    return {"bytes": float(tokens + R * (V * (esz + gsz) + 16 + (8 if case["entropy"] else 0)) + zeros), "flops": 6.0 * R * V}


# ---------------------------------------------------------------- 64 bits

def _moments64(x, case, eps):
    """Mean (0 in the root-mean-square form) and reciprocal deviation of each row."""
    mu = x.mean(1) if case["kind"] == "layer" else torch.zeros_like(x[:, 0])
    var = ((x - mu[:, None]) ** 2).mean(1)
    return mu, 1.0 / torch.sqrt(var + eps)


def exact(case, seed):
    """What run() returns, from the definitions in float64."""
    s = prepare(case, seed)
    T, at = case["tokens"], s["at"]
    zeros = lambda *shape: torch.zeros(shape, dtype=torch.float64, device="cuda")  # noqa: E731
    if case["op"] in ("norm", "norm_bwd"):
        x, gamma = s["x"][at].double(), s["gamma"].double()
        mu, r = _moments64(x, case, s["eps"])
        if case["op"] == "norm":
            y = zeros(T, case["d"])
            y[at] = (x - mu[:, None]) * r[:, None] * gamma + (s["beta"].double() if case["beta"] else 0.0)
            out = {"y": y, "mean": None, "rstd": None}
            if case["stats"]:
                out["rstd"] = zeros(T).index_copy_(0, at, r)
                if case["kind"] == "layer":
                    out["mean"] = zeros(T).index_copy_(0, at, mu)
            return out
        # through the norm's Jacobian: dx = r (I - 11'/d - xh xh'/d) g
        xh, dy = (x - mu[:, None]) * r[:, None], s["dy"][at].double()
        g = dy * gamma
        inner = torch.einsum("ij,ij->i", g, xh) / case["d"]
        dx = g - xh * inner[:, None] - (g.mean(1, keepdim=True) if case["kind"] == "layer" else 0.0)
        full = zeros(T, case["d"])
        full[at] = dx * r[:, None]
        return {"dx": full, "dgamma": torch.einsum("ij,ij->j", dy, xh), "dbeta": dy.sum(0) if case["beta"] else None}

    V, n, k = case["vocab"], at.numel(), case.get("top", 0)
    dense = case["layout"] == "dense"
    if case["op"] == "logprobs":
        out = {"logprob": zeros(T), "entropy": zeros(T), "stats": zeros(T, 2)}
        if k:
            out["top_ids"] = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
            out["top_logprob"] = zeros(T, k)
    else:
        grad = zeros(*s["logits"].shape)
    step = max(1, 60_000_000 // V)
    for i in range(0, n, step):
        t = at[i:i + step]
        rows = t if dense else torch.arange(i, min(n, i + step), device="cuda")
        z, y = s["logits"][rows, :V].double(), s["ids"][t].long()[:, None]
        lp = torch.log_softmax(z, 1)
        p = lp.exp()
        finite = torch.where(p > 0, lp, 0.0)
        H = -(p * finite).sum(1)
        if case["op"] == "logprobs":
            m = z.amax(1)
            out["logprob"][t] = lp.gather(1, y)[:, 0]
            out["entropy"][t] = H
            out["stats"][t] = torch.stack([m, torch.logsumexp(z - m[:, None], 1)], 1)
            if k:
                ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
                out["top_ids"][t] = ids.int()
                out["top_logprob"][t] = lp.gather(1, ids)
            continue
        gl = s["d_logprob"][t, None].double()
        g = -gl * p
        rest = p.scatter(1, y, 0.0).sum(1, keepdim=True)
        g.scatter_(1, y, gl * rest)
        if case["entropy"]:
            g -= s["d_entropy"][t, None].double() * p * (finite + H[:, None])
        grad[rows, :V] = g
    return out if case["op"] == "logprobs" else grad
