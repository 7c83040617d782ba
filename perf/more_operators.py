"""Performance cases of the operators between the token ids and the final norm: embedding lookup and its gradient, the
norms around a block with its gate and residual scale (and their backward pass), and activation checkpoints in 8 bits.

A case is a plain dict.  ``op`` is "embed", "embed_bwd", "block", "block_bwd" or "act8"; common keys:

``tokens``  tokens of the packed batch; ``share`` of them take part (1: no mask), the rest is padding at the ends of
            trajectories
``d``, ``pad``  columns of a row, and elements between the end of one row and the start of the next
``vocab``   rows of the embedding table

The number of tokens that take part follows from the case alone; the seed draws every value and where the padding lies.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

V_MAIN = 151_936
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BYTES = {"bf16": 2, "f32": 4}
CODES = {"e4m3": torch.float8_e4m3fn, "int8": torch.int8}
GROUP = 32  # columns that share one exponent


def listed():
    """Twelve cases: single decoding steps, ordinary batches of each operator, type and layout, and the largest."""
    return [
        # a decoding step of 64 rollouts: one embedding row each, times sqrt(d) as some models have it; latency is all
        dict(name="embed_decode_64", op="embed", tokens=64, share=1.0, vocab=V_MAIN, d=4096, pad=0, w="bf16", out="bf16",
             scale=64.0),
        # the embedding of a packed batch of 8 trajectories
        dict(name="embed_packed", op="embed", tokens=32_768, share=1.0, vocab=V_MAIN, d=5120, pad=0, w="bf16", out="bf16",
             scale=1.0),
        # its gradient over the whole table, which the optimizer then reads: most of it zeros
        dict(name="embed_bwd_packed", op="embed_bwd", tokens=32_768, share=1.0, vocab=V_MAIN, d=4096, pad=0, dout="bf16",
             dw="bf16", scale=1.0),
        # an odd vocabulary and width in fp32, padding at the trajectories' ends
        dict(name="embed_bwd_odd_f32", op="embed_bwd", tokens=8192, share=0.9, vocab=50_001, d=1001, pad=0, dout="f32",
             dw="f32", scale=math.sqrt(1001.0)),
        # a debugging batch of two short trajectories: launches are all it costs
        dict(name="embed_bwd_tiny", op="embed_bwd", tokens=256, share=1.0, vocab=1024, d=256, pad=0, dout="bf16", dw="f32",
             scale=16.0),
        # between two blocks of one token's decoding step
        dict(name="block_decode_1", op="block", tokens=1, share=1.0, d=4096, pad=0, r="bf16", y="bf16", params="bf16",
             kind="rms", post=True, gate="none", resid_scale=1.0, branch_scale=1.0),
        # between two blocks of a packed batch: norm of the block's output, a gate per channel, norm before the next block
        dict(name="block_packed", op="block", tokens=32_768, share=1.0, d=4096, pad=0, r="bf16", y="bf16", params="bf16",
             kind="rms", post=True, gate="channel", resid_scale=1.0, branch_scale=0.25),
        # an fp32 residual stream of an odd width, a gate for every element, layer norms with biases
        dict(name="block_odd_layer_f32", op="block", tokens=4096, share=0.9, d=1001, pad=0, r="f32", y="f32",
             params="f32", kind="layer", post=True, gate="token", resid_scale=0.9, branch_scale=1.0),
        # the way back on a packed batch, activations as they were
        dict(name="block_bwd_packed", op="block_bwd", tokens=16_384, share=1.0, d=5120, pad=0, r="bf16", y="bf16",
             params="bf16", kind="rms", post=True, gate="channel", resid_scale=1.0, branch_scale=0.25, kept="none"),
        # the same from activations that were kept in 8 bits, blocks without a gate
        dict(name="block_bwd_8bit", op="block_bwd", tokens=32_768, share=1.0, d=4096, pad=0, r="bf16", y="bf16",
             params="bf16", kind="rms", post=True, gate="none", resid_scale=1.0, branch_scale=1.0, kept="e4m3"),
        # an activation of a packed batch put away in 8 bits and taken back
        dict(name="act8_packed_e4m3", op="act8", tokens=32_768, share=1.0, d=4096, pad=0, x="bf16", code="e4m3"),
        # a micro-batch of an odd width in fp32, 8-bit whole numbers
        dict(name="act8_odd_int8", op="act8", tokens=512, share=0.9, d=1001, pad=0, x="f32", code="int8"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges."""
    op = rng.choice(("embed", "embed_bwd", "embed_bwd", "block", "block", "block_bwd", "block_bwd", "act8"))
    while True:
        d = _log(rng, 64, 8192)
        d = d if rng.random() < 0.3 else max(64, d // 64 * 64)
        c = dict(op=op, tokens=_log(rng, 1, 32_768), share=rng.choice((1.0, 1.0, round(rng.uniform(0.3, 0.99), 2))), d=d,
                 pad=rng.choice((0, 0, 0, 8, 3)))
        if op in ("embed", "embed_bwd"):
            v = _log(rng, 1024, V_MAIN)
            c.update(vocab=v, scale=rng.choice((1.0, 0.5, math.sqrt(d))))
            if op == "embed":
                c.update(w=rng.choice(("bf16", "f32")), out=rng.choice(("bf16", "bf16", "f32")))
            else:
                c.update(dout=rng.choice(("bf16", "f32")), dw=rng.choice(("bf16", "f32")))
            if v * d > 650_000_000:
                continue
        elif op == "act8":
            c.update(x=rng.choice(("bf16", "bf16", "f32")), code=rng.choice(("e4m3", "int8")))
        else:
            c.update(r=rng.choice(("bf16", "f32")), y=rng.choice(("bf16", "bf16", "f32")), params=rng.choice(("bf16", "f32")),
                     kind=rng.choice(("rms", "layer")), post=rng.random() < 0.6, gate=rng.choice(("none", "channel", "token")),
                     resid_scale=rng.choice((1.0, 1.0, 0.9)), branch_scale=rng.choice((1.0, 0.25)))
            if op == "block_bwd":
                c["kept"] = rng.choice(("none", "none", "e4m3", "int8"))
        if _taking_part(c) < 1 or c["tokens"] * d > 140_000_000:
            continue
        return c


# ---------------------------------------------------------------- inputs

def _taking_part(case):
    return case["tokens"] if case["share"] >= 1.0 else int(round(case["share"] * case["tokens"]))


def _generator(seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return gen


def _mask(case, seed):
    """Trajectories of about 2,000 tokens, each padded at its end; the right number of tokens, turned by the seed."""
    T, n = case["tokens"], _taking_part(case)
    if case["share"] >= 1.0:
        return None, torch.arange(T, device="cuda")
    rng = np.random.default_rng([T, n])
    m = np.zeros(T, np.uint8)
    runs = max(1, T // 2000)
    cut = lambda total: np.diff(np.concatenate([[0], np.sort(rng.integers(0, total + 1, runs - 1)), [total]]))  # noqa: E731
    at = 0
    for on, off in zip(cut(n), cut(T - n)):
        m[at:at + on] = 1
        at += on + off
    m = np.roll(m, int(np.random.default_rng(seed).integers(0, T)))
    return torch.from_numpy(m).cuda(), torch.from_numpy(np.nonzero(m)[0]).cuda()


def _stream(gen, T, d):
    """Values of a residual stream: a few channels many times as large as the others, a mean that is not 0."""
    scale = torch.where(torch.rand(d, generator=gen, device="cuda") < 0.01, 30.0, 1.0)
    return torch.randn((T, d), generator=gen, device="cuda") * scale + 0.3


def _stats(s, resid, y):
    """What the forward pass keeps of each row: mu and r of the block's output, mu and r of the new residual stream."""
    c, at = s["case"], s["at"]
    out = torch.zeros((c["tokens"], 4), dtype=torch.float32, device="cuda")
    for k, v, on in ((0, y, c["post"]), (2, resid, True)):
        if on:
            v = v[at].double()
            mu = v.mean(1) if c["kind"] == "layer" else torch.zeros(at.numel(), dtype=torch.float64, device="cuda")
            out[at, k] = mu.float()
            out[at, k + 1] = ((v - mu[:, None]).square().mean(1) + s["eps"]).rsqrt().float()
    return out


def _power(k):
    """2^k in fp32 from its bits, k in -126 .. 127 (-127: 0)."""
    return ((k + 127) << 23).view(torch.float32)


def _largest(x):
    """The largest magnitude of each group of columns."""
    T, d = x.shape
    n = (d + GROUP - 1) // GROUP
    return torch.nn.functional.pad(x, (0, n * GROUP - d)).view(T, n, GROUP).abs().amax(2)


def _encode(x, code):
    """Codes, and one exponent byte per group, of fp32 values.  A group's exponent is the smallest power of two that brings its
    largest value within the codes' range; it scales without rounding."""
    top = 448.0 if code == "e4m3" else 127.0
    m, e = torch.frexp(_largest(x))
    mt, et = math.frexp(top)
    k = torch.clamp(e - et + (m > mt).int(), min=-126)
    k = torch.where(m == 0, -126, k)
    v = x * _power(-k).repeat_interleave(GROUP, 1)[:, :x.shape[1]]
    q = v.to(torch.float8_e4m3fn) if code == "e4m3" else torch.round(v).to(torch.int8)
    return q, (k + 127).to(torch.uint8)


def _decode(q, exps):
    return q.float() * _power(exps.int() - 127).repeat_interleave(GROUP, 1)[:, :q.shape[1]]


def _rows_of(q, at):
    """Some rows of codes (indexing takes no 8-bit floats)."""
    return q.view(torch.uint8)[at].view(q.dtype)


def prepare(case, seed):
    """What a program holds before the call: the inputs, and the buffers that the outputs go to."""
    mask, at = _mask(case, seed)
    s = dict(case=case, mask=mask, at=at, eps=1e-6, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    T, d, gen = case["tokens"], case["d"], _generator(seed)
    rand = lambda *shape: torch.randn(shape, generator=gen, device="cuda")  # noqa: E731

    def rows(t, values=None, n=T):
        out = torch.zeros((n, d + case["pad"]), dtype=CODES[t] if t in CODES else TYPES[t], device="cuda")[:, :d]
        return out if values is None else out.copy_(values)

    if case["op"] in ("embed", "embed_bwd"):
        V = case["vocab"]
        # frequencies as 1 / rank; the first few ids (a chat template's) are every tenth token or so
        rank = torch.exp(torch.rand(T, generator=gen, device="cuda") * math.log(V)).long().clamp_(1, V) - 1
        s["ids"] = torch.randperm(V, generator=gen, device="cuda")[rank].int()
        if case["op"] == "embed":
            s["w"] = rows(case["w"], n=V)
            for i in range(0, V, 16_384):
                n = min(16_384, V - i)
                s["w"][i:i + n] = 0.02 * rand(n, d)
            s["out"] = rows(case["out"])
        else:
            s["dout"] = rows(case["dout"], 1e-3 * rand(T, d))
            s["dw"] = rows(case["dw"], n=V)
        return s
    if case["op"] == "act8":
        s["x"] = rows(case["x"], _stream(gen, T, d))
        s["out"], s["codes"] = rows(case["x"]), rows(case["code"])
        s["exps"] = torch.zeros((T, (d + GROUP - 1) // GROUP), dtype=torch.uint8, device="cuda")
        return s
    P = TYPES[case["params"]]
    layer = case["kind"] == "layer"
    vector = lambda mean, dev: (mean + dev * rand(d)).to(P)  # noqa: E731
    s["gamma_pre"], s["beta_pre"] = vector(1.0, 0.2), vector(0.0, 0.1) if layer else None
    s["gamma_post"] = vector(1.0, 0.2) if case["post"] else None
    s["beta_post"] = vector(0.0, 0.1) if case["post"] and layer else None
    s["gate"] = vector(0.5, 0.2) if case["gate"] == "channel" else \
        rows(case["y"], torch.sigmoid(rand(T, d))) if case["gate"] == "token" else None
    resid, y = rows(case["r"], _stream(gen, T, d)), rows(case["y"], 0.5 * _stream(gen, T, d))
    if case["op"] == "block":
        s.update(resid=resid, y=y, resid_out=rows(case["r"]), h=rows(case["y"]))
        s["stats"] = torch.zeros((T, 4), dtype=torch.float32, device="cuda")
        return s
    s["stats"] = _stats(s, resid, y)
    for name, v in (("resid", resid), ("y", y)):
        if case["kept"] == "none":
            s[name] = v
        else:
            q, exps = _encode(v.float(), case["kept"])
            s[name] = (rows(case["kept"]).copy_(q), exps)
    s["dh"], s["d_resid_out"] = rows(case["y"], 1e-3 * rand(T, d)), rows(case["r"], 1e-3 * rand(T, d))
    s["d_resid"], s["dy"] = rows(case["r"]), rows(case["y"])
    total = lambda on: torch.zeros(d, dtype=torch.float32, device="cuda") if on else None  # noqa: E731
    s["dgamma_pre"], s["dbeta_pre"] = total(True), total(layer)
    s["dgamma_post"], s["dbeta_post"] = total(case["post"]), total(case["post"] and layer)
    s["dgate"] = rows(case["y"]) if case["gate"] == "token" else total(case["gate"] == "channel")
    return s


# ---------------------------------------------------------------- a pass

GRADS = ("d_resid", "dy", "dgate", "dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre")


def run(s):
    return _own(s) if own else PLAIN[s["case"]["op"]](s)


def _own(s):
    import paper_2607_05804_gb300 as lib

    c = s["case"]
    if c["op"] == "embed":
        lib.turnopd_embedding_fwd(s["w"], s["ids"], s["mask"], c["scale"], s["out"], s["status"])
        return s["out"]
    if c["op"] == "embed_bwd":
        if "workspace" not in s:
            s["workspace"] = torch.empty(lib.turnopd_embedding_bwd_workspace_bytes(c["tokens"], c["d"], c["vocab"]),
                                         dtype=torch.uint8, device="cuda")
        lib.turnopd_embedding_bwd(s["dout"], s["ids"], s["mask"], c["scale"], s["dw"], 0, s["workspace"], s["status"])
        return s["dw"]
    if c["op"] == "act8":
        lib.turnopd_act8_store(s["x"], s["mask"], s["codes"], s["exps"], s["status"])
        lib.turnopd_act8_load(s["codes"], s["exps"], s["out"])
        return s["out"]
    kind = lib.TURNOPD_RMS_NORM if c["kind"] == "rms" else lib.TURNOPD_LAYER_NORM
    if c["op"] == "block":
        lib.turnopd_block_norm_fwd(s["resid"], s["y"], s["gamma_post"], s["beta_post"], s["gate"], s["gamma_pre"],
                                   s["beta_pre"], s["mask"], kind, s["eps"], c["resid_scale"], c["branch_scale"],
                                   s["resid_out"], s["h"], s["stats"], s["status"])
        return {k: s[k] for k in ("resid_out", "h", "stats")}
    if "workspace" not in s:
        s["workspace"] = torch.empty(lib.turnopd_block_norm_bwd_workspace_bytes(c["tokens"], c["d"]), dtype=torch.uint8,
                                     device="cuda")
    lib.turnopd_block_norm_bwd(s["resid"], s["y"], s["gamma_post"], s["beta_post"], s["gate"], s["gamma_pre"], s["mask"], kind,
                               c["resid_scale"], c["branch_scale"], s["stats"], s["dh"], s["d_resid_out"], s["d_resid"],
                               s["dy"], s["dgate"], s["dgamma_post"], s["dbeta_post"], s["dgamma_pre"], s["dbeta_pre"],
                               s["workspace"])
    return {k: s[k] for k in GRADS}


def _take(s, v):
    """The rows that take part, in 32 bits."""
    return (v if s["mask"] is None else v[s["at"]]).float()


def _put(s, to, v):
    """Rows of results to their tokens, zeros to the others."""
    if s["mask"] is None:
        to.copy_(v)
    else:
        to.zero_()
        to[s["at"]] = v.to(to.dtype)


def _plain_embed(s):
    ids = s["ids"][s["at"]].long()
    _put(s, s["out"], s["w"][ids].float() * s["case"]["scale"])
    return s["out"]


def _plain_embed_bwd(s):
    c = s["case"]
    total = torch.zeros((c["vocab"], c["d"]), dtype=torch.float32, device="cuda")
    total.index_add_(0, s["ids"][s["at"]].long(), _take(s, s["dout"]))
    s["dw"].copy_(total.mul_(c["scale"]))
    return s["dw"]


def _plain_act8(s):
    x = _take(s, s["x"])
    q, exps = _encode(x, s["case"]["code"])
    _put(s, s["codes"].view(torch.int8), q.view(torch.int8))
    s["exps"].zero_()
    s["exps"][s["at"]] = exps
    s["out"].copy_(_decode(s["codes"], s["exps"]))
    return s["out"]


def _norm(x, gamma, beta, kind, eps):
    mu = x.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(x[:, :1])
    x = x - mu
    r = (x.square().mean(1, keepdim=True) + eps).rsqrt()
    out = x * r * gamma.float()
    return mu, r, out if beta is None else out + beta.float()


def _plain_block(s):
    c = s["case"]
    b, kept = _take(s, s["y"]), torch.zeros((s["at"].numel(), 4), dtype=torch.float32, device="cuda")
    if c["post"]:
        kept[:, 0:1], kept[:, 1:2], b = _norm(b, s["gamma_post"], s["beta_post"], c["kind"], s["eps"])
    if c["gate"] == "channel":
        b = b * s["gate"].float()
    elif c["gate"] == "token":
        b = b * _take(s, s["gate"])
    resid = c["resid_scale"] * _take(s, s["resid"]) + c["branch_scale"] * b
    kept[:, 2:3], kept[:, 3:4], h = _norm(resid, s["gamma_pre"], s["beta_pre"], c["kind"], s["eps"])
    _put(s, s["resid_out"], resid)
    _put(s, s["h"], h)
    _put(s, s["stats"], kept)
    return {k: s[k] for k in ("resid_out", "h", "stats")}


def _plain_block_bwd(s):
    c, at = s["case"], s["at"]
    layer = c["kind"] == "layer"
    kept = s["stats"][at]
    if c["kept"] == "none":
        resid, y = _take(s, s["resid"]), _take(s, s["y"])
    else:
        resid, y = (_decode(_rows_of(q, at), e[at]) for q, e in (s["resid"], s["y"]))

    def back(g, xh, r):
        out = g - xh * (g * xh).mean(1, keepdim=True)
        if layer:
            out -= g.mean(1, keepdim=True)
        return out * r

    xh = (resid - kept[:, 2:3]) * kept[:, 3:4]
    dh = _take(s, s["dh"])
    s["dgamma_pre"].copy_((dh * xh).sum(0))
    if layer:
        s["dbeta_pre"].copy_(dh.sum(0))
    D = _take(s, s["d_resid_out"]) + back(dh * s["gamma_pre"].float(), xh, kept[:, 3:4])
    _put(s, s["d_resid"], c["resid_scale"] * D)
    xh = (y - kept[:, 0:1]) * kept[:, 1:2] if c["post"] else y
    b = xh * s["gamma_post"].float() if c["post"] else y
    if s["beta_post"] is not None:
        b = b + s["beta_post"].float()
    D = c["branch_scale"] * D
    E = D
    if c["gate"] == "channel":
        s["dgate"].copy_((D * b).sum(0))
        E = D * s["gate"].float()
    elif c["gate"] == "token":
        _put(s, s["dgate"], D * b)
        E = D * _take(s, s["gate"])
    if c["post"]:
        s["dgamma_post"].copy_((E * xh).sum(0))
        if layer:
            s["dbeta_post"].copy_(E.sum(0))
        E = back(E * s["gamma_post"].float(), xh, kept[:, 1:2])
    _put(s, s["dy"], E)
    return {k: s[k] for k in GRADS}


PLAIN = {"embed": _plain_embed, "embed_bwd": _plain_embed_bwd, "act8": _plain_act8, "block": _plain_block,
         "block_bwd": _plain_block_bwd}


# ---------------------------------------------------------------- what a pass needs

def work(case):
    T, R, d = case["tokens"], _taking_part(case), case["d"]
    mask = T if case["share"] < 1.0 else 0
    if case["op"] == "embed":
        # the table's rows that R tokens name, each read once: rank i has log((i + 2) / (i + 1)) / log(vocab) of the tokens
        p = np.log1p(1.0 / np.arange(1, case["vocab"])) / math.log(case["vocab"])
        distinct = float(-np.expm1(R * np.log1p(-p)).sum())
        return {"bytes": float(mask + 4 * R + distinct * d * BYTES[case["w"]] + T * d * BYTES[case["out"]]), "flops": 1.0 * R * d}
    if case["op"] == "embed_bwd":
        return {"bytes": float(mask + 4 * R + R * d * BYTES[case["dout"]] + case["vocab"] * d * BYTES[case["dw"]]),
                "flops": 2.0 * R * d}
    codes = d + (d + GROUP - 1) // GROUP
    if case["op"] == "act8":
        return {"bytes": float(mask + R * d * BYTES[case["x"]] + 2 * T * codes + T * d * BYTES[case["x"]]), "flops": 4.0 * R * d}
    r, y, p = BYTES[case["r"]], BYTES[case["y"]], BYTES[case["params"]]
    gate = d * y if case["gate"] == "token" else 0
    vectors = 1 + case["post"] + (case["kind"] == "layer") * (1 + case["post"]) + (case["gate"] == "channel")
    if case["op"] == "block":
        return {"bytes": float(mask + R * (d * (r + y) + gate) + T * (d * (r + y) + 16) + vectors * d * p), "flops": 16.0 * R * d}
    kept = d * (r + y) if case["kept"] == "none" else 2 * codes
    return {"bytes": float(mask + R * (kept + d * (r + y) + gate + 16) + T * (d * (r + y) + gate) + vectors * d * (p + 4)),
            "flops": 32.0 * R * d}


# ---------------------------------------------------------------- 64 bits

def _code_values(x, code):
    """What the codes of each group stand for, from the definition of the two formats, on doubles."""
    T, d = x.shape
    out = torch.empty_like(x)
    power = lambda k: ((k.long() + 1023) << 52).view(torch.float64)  # noqa: E731
    top = 448.0 if code == "e4m3" else 127.0
    for j in range(0, d, GROUP):
        v = x[:, j:j + GROUP]
        most = v.abs().amax(1, keepdim=True)
        k = torch.ceil(torch.log2(most / top)).clamp_(min=-125.0)
        k = torch.where(top * power(k - 1) >= most, k - 1, k)
        unit = power(k)
        if code == "e4m3":  # four significant bits, the last at 2^-9 at least
            unit = unit * power(torch.frexp((v / unit).abs().clamp_(min=2.0 ** -6)).exponent - 4)
        out[:, j:j + GROUP] = torch.round(v / unit) * unit
    return out


def _code_worth(q, exps, code):
    """The values of given codes, from their bits."""
    b = q.contiguous().view(torch.uint8).long()
    if code == "int8":
        v = torch.where(b > 127, b - 256, b).double()
    else:
        e, m = (b >> 3) & 15, (b & 7).double()
        v = torch.where(e > 0, (8 + m) * torch.exp2(e.double() - 10), m * 2.0 ** -9) * (1 - 2 * (b >> 7)).double()
    return v * torch.exp2(exps.double() - 127).repeat_interleave(GROUP, 1)[:, :q.shape[1]]


def exact(case, seed):
    """What run() returns, from the definitions in float64."""
    s = prepare(case, seed)
    T, d, at = case["tokens"], case["d"], s["at"]

    def full(v, n=T):
        out = torch.zeros((n, v.shape[1]), dtype=torch.float64, device="cuda")
        out[at] = v
        return out

    if case["op"] == "embed":
        return full(case["scale"] * torch.nn.functional.embedding(s["ids"][at].long(), s["w"]).double())
    if case["op"] == "embed_bwd":
        dw = torch.zeros((case["vocab"], d), dtype=torch.float64, device="cuda")
        uniq, inv = torch.unique(s["ids"][at].long(), return_inverse=True)
        sums = torch.zeros((uniq.numel(), d), dtype=torch.float64, device="cuda")
        sums.scatter_add_(0, inv[:, None].expand(-1, d), s["dout"][at].double())
        dw[uniq] = sums * case["scale"]
        return dw
    if case["op"] == "act8":
        return full(_code_values(s["x"][at].double(), case["code"]))

    def moments(x):
        mu = x.mean(1, keepdim=True) if case["kind"] == "layer" else torch.zeros_like(x[:, :1])
        return mu, 1.0 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + s["eps"])

    wide = lambda v: None if v is None else v.double()  # noqa: E731
    g1, b1, g2, b2 = (wide(s[k]) for k in ("gamma_post", "beta_post", "gamma_pre", "beta_pre"))
    gate = 1.0 if s["gate"] is None else s["gate"].double() if case["gate"] == "channel" else s["gate"][at].double()
    gate = case["branch_scale"] * gate
    if case["op"] == "block":
        y, kept = s["y"][at].double(), torch.zeros((at.numel(), 4), dtype=torch.float64, device="cuda")
        if case["post"]:
            mu, r = moments(y)
            kept[:, 0:1], kept[:, 1:2] = mu, r
            y = (y - mu) * r * g1 + (0.0 if b1 is None else b1)
        resid = torch.addcmul(case["resid_scale"] * s["resid"][at].double(), y, torch.as_tensor(gate, device="cuda", dtype=torch.float64))
        mu, r = moments(resid)
        kept[:, 2:3], kept[:, 3:4] = mu, r
        h = (resid - mu) * r * g2 + (0.0 if b2 is None else b2)
        return {"resid_out": full(resid), "h": full(h), "stats": full(kept)}

    def activation(v):
        return v[at].double() if case["kept"] == "none" else _code_worth(_rows_of(v[0], at), v[1][at], case["kept"])

    def through(g, x, k):
        """The norm's Jacobian, transposed, from the statistics that were kept."""
        xh = (x - kept[:, k:k + 1]) * kept[:, k + 1:k + 2]
        inner = torch.einsum("ij,ij->i", g, xh)[:, None] / d
        out = g - inner * xh
        return xh, kept[:, k + 1:k + 2] * (out - g.mean(1, keepdim=True) if case["kind"] == "layer" else out)

    kept = s["stats"][at].double()
    dh, y = s["dh"][at].double(), activation(s["y"])
    xh, dx = through(dh * g2, activation(s["resid"]), 2)
    out = {"dgamma_pre": torch.einsum("ij,ij->j", dh, xh), "dbeta_pre": dh.sum(0) if case["kind"] == "layer" else None}
    D = s["d_resid_out"][at].double() + dx
    E = gate * D
    out.update(d_resid=full(case["resid_scale"] * D), dgate=None, dgamma_post=None, dbeta_post=None)
    b = y
    if case["post"]:
        xh, dy = through(E * g1, y, 0)
        b = xh * g1 + (0.0 if b1 is None else b1)
        out["dgamma_post"] = torch.einsum("ij,ij->j", E, xh)
        out["dbeta_post"] = E.sum(0) if case["kind"] == "layer" else None
    out["dy"] = full(dy if case["post"] else E)
    if case["gate"] == "channel":
        out["dgate"] = case["branch_scale"] * torch.einsum("ij,ij->j", D, b)
    elif case["gate"] == "token":
        out["dgate"] = full(case["branch_scale"] * D * b)
    return {k: out[k] for k in GRADS}
