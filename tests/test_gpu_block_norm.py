"""The norms around a block with its gate and residual connection, and their backward pass, against float64.

Tolerances.  A norm's xh is off by 1e-5 (1 + |xh| + |mu| rho), as derived for the norm before the LM head: fp32 sums of d terms,
at most d / 32 of them in one partial sum, and x - mu rounded once.  What r' is off by (t) moves a later h by
rho (t_j + (1 + |xh|) rms t) through x - mu, mu and rho.  Going back, every result is a sum of terms each good to 2e-5 of the
magnitudes it is made of.  Outputs are rounded once: half a step of their type.  Sums over the tokens: at most 335 terms to a
partial sum, so 2e-5 of the sum of their magnitudes too.
"""
import pytest
import torch

import paper_2607_05804_gb300 as P

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
LAYER, RMS = P.TURNOPD_LAYER_NORM, P.TURNOPD_RMS_NORM
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
VECTORS = ("dgamma_post", "dbeta_post", "dgamma_pre", "dbeta_pre")


def strided(T, d, ld, offset, dtype, fill=3.0):
    return torch.full((T * ld + offset,), fill, device="cuda", dtype=dtype)[offset:].view(T, ld)[:, :d]


def half_step(t):
    return torch.finfo(t).eps / 2


def within(a, b, tol, what=""):
    err = (a.double() - b).abs()
    assert bool(torch.isfinite(a.double()).all()), what
    assert bool((err <= tol).all()), (what, float((err / tol.clamp(min=1e-300)).max()))


class Case:
    def __init__(self, T, d, rdt=BF, ydt=BF, pdt=BF, kind=RMS, post=True, pre=True, gate="none", beta=None, alpha=1.0, s=1.0,
                 ld=None, offset=0, seed=0, masked=0.0, eps=1e-6):
        self.g = torch.Generator(device="cuda").manual_seed(seed + 7 * d + T)
        self.T, self.d, self.rdt, self.ydt, self.kind, self.alpha, self.s, self.eps = T, d, rdt, ydt, kind, alpha, s, eps
        self.ld, self.offset = ld or d, offset
        rand = lambda *shape: torch.randn(shape, generator=self.g, device="cuda")  # noqa: E731
        scale = torch.where(torch.rand(d, generator=self.g, device="cuda") < 0.02, 25.0, 1.0)
        self.resid = self.rows(rdt).copy_(rand(T, d) * scale + 0.5)
        self.y = self.rows(ydt).copy_(rand(T, d) * scale * 0.7 - 0.2)
        beta = kind == LAYER if beta is None else beta
        vec = lambda m, v: (m + v * rand(d)).to(pdt)  # noqa: E731
        self.gamma_post, self.beta_post = (vec(1, 0.3), vec(0, 0.2) if beta else None) if post else (None, None)
        self.gamma_pre, self.beta_pre = (vec(1, 0.3), vec(0, 0.2) if beta else None) if pre else (None, None)
        self.gate = vec(0.5, 0.3) if gate == "channel" else self.rows(ydt).copy_(torch.sigmoid(rand(T, d))) if gate == "token" else None
        self.channel = gate == "channel"
        self.mask = (torch.rand(T, generator=self.g, device="cuda") >= masked).to(torch.uint8) if masked else None
        self.on = torch.ones(T, dtype=torch.bool, device="cuda") if self.mask is None else self.mask.bool()
        self.dh = self.rows(ydt).copy_(rand(T, d)) if pre else None
        self.d_resid_out = self.rows(rdt).copy_(rand(T, d))
        for t in (self.resid, self.y, self.dh, self.d_resid_out, self.gate if gate == "token" else None):
            if t is not None and self.mask is not None:
                t[~self.on] = float("nan")  # rows of masked tokens are not read

    def rows(self, dtype, fill=3.0):
        return strided(self.T, self.d, self.ld, self.offset, dtype, fill)

    def forward(self, resid_out=None, stream=None):
        resid_out = self.rows(self.rdt) if resid_out is None else resid_out
        h = self.rows(self.ydt) if self.gamma_pre is not None else None
        stats, st = torch.full((self.T, 4), 7.0, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        P.turnopd_block_norm_fwd(self.resid, self.y, self.gamma_post, self.beta_post, self.gate, self.gamma_pre, self.beta_pre,
                                 self.mask, self.kind, self.eps, self.alpha, self.s, resid_out, h, stats, st, stream)
        return resid_out, h, stats, st

    def moments(self, x):
        mu = x.mean(1, keepdim=True) if self.kind == LAYER else torch.zeros_like(x[:, :1])
        r = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + self.eps)
        return mu, r, (x - mu) * r

    def wide(self, t):
        return t if t is None or not torch.is_tensor(t) else t.double()

    def gate64(self):
        g = 1.0 if self.gate is None else self.gate.double() if self.channel else self.gate[self.on].double()
        return self.s * g

    def formula(self, resid, y):
        """(r', h, stats, b) in float64, differentiable."""
        b, kept = y, [torch.zeros_like(y[:, :1])] * 4
        if self.gamma_post is not None:
            kept[0], kept[1], xh = self.moments(y)
            b = xh * self.wide(self.gamma_post) + (self.wide(self.beta_post) if self.beta_post is not None else 0.0)
        out = self.alpha * resid + self.gate64() * b
        h = None
        if self.gamma_pre is not None:
            kept[2], kept[3], xh = self.moments(out)
            h = xh * self.wide(self.gamma_pre) + (self.wide(self.beta_pre) if self.beta_pre is not None else 0.0)
        return out, h, torch.cat(kept, 1), b

    def check_forward(self, resid_out, h, stats, st):
        assert st.item() == 0
        on = self.on
        resid, y = self.resid[on].double(), self.y[on].double()
        out, h64, kept, b = self.formula(resid, y)
        t_b = 0.0
        if self.gamma_post is not None:
            xh = (y - kept[:, 0:1]) * kept[:, 1:2]
            t_b = 1e-5 * (1 + xh.abs() + kept[:, 0:1].abs() * kept[:, 1:2]) * self.gamma_post.double().abs()
        g = self.gate64() if torch.is_tensor(self.gate64()) else torch.full((), self.gate64(), dtype=torch.float64, device="cuda")
        t_r = g.abs() * (t_b + 2.0 ** -22 * b.abs()) + 2.0 ** -22 * (self.alpha * resid).abs()
        within(resid_out[on], out, t_r + half_step(self.rdt) * out.abs() + 1e-38, "resid_out")
        if h is not None:
            mu, r = kept[:, 2:3], kept[:, 3:4]
            xh = (out - mu) * r
            t = 1e-5 * (1 + xh.abs() + mu.abs() * r) + r * (t_r + (1 + xh.abs()) * (t_r ** 2).mean(1, keepdim=True).sqrt())
            within(h[on], h64, t * self.gamma_pre.double().abs() + 1e-6 * h64.abs() + half_step(self.ydt) * h64.abs() + 1e-38, "h")
            assert not h[~on].any()
        rms = torch.stack([y.abs().mean(1), kept[:, 1], (out.abs() + 10 * t_r).mean(1), kept[:, 3]], 1)
        rel = torch.stack([torch.ones_like(kept[:, 0]), 1 + kept[:, 0].abs() * kept[:, 1], torch.ones_like(kept[:, 0]),
                           1 + (kept[:, 2].abs() + 1e5 * (t_r ** 2).mean(1).sqrt()) * kept[:, 3]], 1)
        within(stats[on], kept, 1e-5 * rms * rel + 1e-30, "stats")
        assert not resid_out[~on].any() and not stats[~on].any()

    # -------------------------------------------------------- back

    def kept(self, x, code):
        if code is None:
            return x
        q = torch.zeros((self.T, self.ld), dtype=torch.uint8, device="cuda").view(code)[:, :self.d]
        exps, st = torch.zeros((self.T, (self.d + 31) // 32), dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        P.turnopd_act8_store(x, self.mask, q, exps, st)
        assert st.item() == 0
        return q, exps

    def values(self, x):
        if torch.is_tensor(x):
            return x[self.on].double()
        out = torch.empty((self.T, self.d), device="cuda")
        P.turnopd_act8_load(*x, out)
        return out[self.on].double()

    def backward(self, resid, y, stats, in_place=False, skip=(), stream=None, d_resid_out="own"):
        f32 = lambda on: torch.full((self.d,), 5.0, device="cuda") if on else None  # noqa: E731
        dro = self.d_resid_out if isinstance(d_resid_out, str) else d_resid_out
        o = dict(d_resid=dro if in_place else self.rows(self.rdt), dy=self.rows(self.ydt),
                 dgate=None if self.gate is None else f32(True) if self.channel else self.rows(self.ydt),
                 dgamma_post=f32(self.gamma_post is not None), dbeta_post=f32(self.gamma_post is not None),
                 dgamma_pre=f32(self.gamma_pre is not None), dbeta_pre=f32(self.gamma_pre is not None))
        o.update({k: None for k in skip})
        ws = torch.full((P.turnopd_block_norm_bwd_workspace_bytes(self.T, self.d),), 255, dtype=torch.uint8, device="cuda")
        P.turnopd_block_norm_bwd(resid, y, self.gamma_post, self.beta_post, self.gate, self.gamma_pre, self.mask, self.kind,
                                 self.alpha, self.s, stats, self.dh, dro, o["d_resid"], o["dy"], o["dgate"], o["dgamma_post"],
                                 o["dbeta_post"], o["dgamma_pre"], o["dbeta_pre"], ws, stream)
        return o

    def check_backward(self, o, resid, y, stats, dro="own"):
        """From the formulas, with the magnitudes that each result is made of beside it."""
        on = self.on
        layer = 1.0 if self.kind == LAYER else 0.0
        stats = stats[on].double()
        dro = self.d_resid_out if isinstance(dro, str) else dro
        D = torch.zeros((int(on.sum()), self.d), dtype=torch.float64, device="cuda") if dro is None else dro[on].double()
        mD = D.abs()

        def through(g, mg, x, mu, r):
            xh = (x - mu) * r
            mean = lambda v: v.mean(1, keepdim=True)  # noqa: E731
            return (r * (g - layer * mean(g) - xh * mean(g * xh)),
                    r * (mg + layer * mean(mg) + xh.abs() * mean(mg * xh.abs())), xh)

        if self.gamma_pre is not None:
            dh = self.dh[on].double()
            g = dh * self.gamma_pre.double()
            a, m, xh = through(g, g.abs(), self.values(resid), stats[:, 2:3], stats[:, 3:4])
            D, mD = D + a, mD + m
            self.total(o["dgamma_pre"], dh * xh, (dh * xh).abs(), "dgamma_pre")
            self.total(o["dbeta_pre"], dh, dh.abs(), "dbeta_pre")
        self.rows_close(o["d_resid"], self.alpha * D, abs(self.alpha) * mD, self.rdt, "d_resid")
        gate = self.gate64()
        E = gate * D
        mE = (gate.abs() if torch.is_tensor(gate) else abs(gate)) * mD
        if self.gamma_post is not None:
            gp = self.gamma_post.double()
            a, m, xh = through(E * gp, mE * gp.abs(), self.values(y), stats[:, 0:1], stats[:, 1:2])
            self.rows_close(o["dy"], a, m, self.ydt, "dy")
            self.total(o["dgamma_post"], E * xh, mE * xh.abs(), "dgamma_post")
            self.total(o["dbeta_post"], E, mE, "dbeta_post")
            b = xh * gp
            mb = b.abs() + (self.beta_post.double().abs() if self.beta_post is not None else 0.0)
            b = b + (self.beta_post.double() if self.beta_post is not None else 0.0)
        else:
            self.rows_close(o["dy"], E, mE, self.ydt, "dy")
            b = self.values(y) if o["dgate"] is not None else None
            mb = b.abs() if b is not None else None
        if o["dgate"] is not None and self.channel:
            self.total(o["dgate"], self.s * D * b, abs(self.s) * mD * mb, "dgate")
        elif o["dgate"] is not None:
            self.rows_close(o["dgate"], self.s * D * b, abs(self.s) * mD * mb, self.ydt, "dgate")

    def rows_close(self, got, want, size, dtype, what):
        if got is not None:
            within(got[self.on], want, 2e-5 * size + half_step(dtype) * want.abs() + 1e-37, what)
            assert not got[~self.on].any(), what

    def total(self, got, terms, size, what):
        if got is not None:
            within(got, terms.sum(0), 2e-5 * size.sum(0) + 1e-37, what)


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (4, 31), (9, 128), (70, 255), (5, 1000), (33, 1001), (400, 1024), (3, 2048), (2, 4095),
          (1, 4096), (310, 4096), (7, 5120), (3, 8192), (2, 8200), (2, 20001)]
LAYOUTS = [(BF, BF, BF, 0, 0), (F, BF, F, 0, 0), (F, F, BF, 8, 0), (BF, F, F, 3, 1), (BF, BF, F, 8, 8)]


def case(T, d, layout, **kw):
    rdt, ydt, pdt, pad, off = layout
    return Case(T, d, rdt, ydt, pdt, ld=d + pad, offset=off, **kw)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward_and_backward(T, d, kind):
    for k, layout in enumerate(LAYOUTS):
        for gate in ("none", "channel", "token"):
            c = case(T, d, layout, kind=kind, gate=gate, alpha=(1.0, 0.7)[k % 2], s=(1.0, 0.25)[k % 2])
            out = c.forward()
            c.check_forward(*out)
            resid, stats = out[0], out[2]
            o = c.backward(resid, c.y, stats)
            c.check_backward(o, resid, c.y, stats)


@pytest.mark.parametrize("post,pre", [(False, True), (True, False), (False, False)])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("d,pad,off", [(264, 0, 0), (1001, 0, 0), (2048, 8, 0), (9000, 0, 0)])
def test_with_one_norm_or_none(d, pad, off, gate, post, pre):
    for kind, beta in ((LAYER, False), (RMS, True)):
        c = case(50, d, (BF, BF, F, pad, off), kind=kind, beta=beta, post=post, pre=pre, gate=gate, alpha=-0.5, s=2.0, masked=0.3)
        out = c.forward()
        c.check_forward(*out)
        # what nothing needs may be missing
        resid = out[0] if pre else None
        y = c.y if post or gate != "none" else None
        o = c.backward(resid, y, out[2] if post or pre else None)
        c.check_backward(o, resid, y, out[2])
        if pre:  # nothing comes back through the stream
            o = c.backward(resid, y, out[2], d_resid_out=None)
            c.check_backward(o, resid, y, out[2], dro=None)


@pytest.mark.parametrize("d", [63, 511, 1001, 1537, 2047, 2601, 4100, 5119, 7003, 8191, 256, 640, 2560, 6144, 8192])
def test_many_rows_masks_and_in_place(d):
    """Rows enough for several to each block, of any alignment, with a mask; r' over r and dr over dr'."""
    T = 1300
    for k, (layout, gate, kind) in enumerate((((BF, BF, BF, 0, 0), "channel", RMS), ((F, BF, F, 1, 1), "none", LAYER),
                                              ((BF, F, F, 8 - d % 8, 0), "token", RMS))):
        c = case(T, d, layout, kind=kind, gate=gate, masked=0.4, seed=k)
        ref = c.forward()
        c.check_forward(*ref)
        old = c.resid.clone()
        got = c.forward(resid_out=c.resid)
        assert all(torch.equal(a, b) for a, b in zip(ref, got) if a is not None)
        c.resid = old
        o = c.backward(ref[0], c.y, ref[2])
        c.check_backward(o, ref[0], c.y, ref[2])
        p = c.backward(ref[0], c.y, ref[2], in_place=True)
        for name in o:
            assert o[name] is None or torch.equal(o[name], p[name]), name


@pytest.mark.parametrize("d", [64, 1001, 4096])
def test_arrays_of_different_strides(d):
    """Rows that begin at different elements in different arrays: the results are the same numbers."""
    for gate, kind in (("channel", RMS), ("token", LAYER)):
        c = case(150, d, (BF, BF, F, 0, 0), gate=gate, kind=kind, masked=0.2)
        c.y = strided(150, d, d + 3, 1, BF).copy_(c.y)
        out = c.forward()
        c.check_forward(*out)
        c.dh = strided(150, d, d + 5, 0, BF).copy_(c.dh)
        o = c.backward(out[0], c.y, out[2])
        c.check_backward(o, out[0], c.y, out[2])


@pytest.mark.parametrize("code", [E4M3, INT8])
@pytest.mark.parametrize("T,d,pad", [(1, 32, 0), (5, 33, 0), (40, 1001, 0), (300, 4096, 0), (300, 4096, 16), (200, 5120, 0), (7, 8192, 0),
                                     (3, 9000, 0), (64, 520, 0), (64, 520, 3)])
def test_backward_from_8_bits(T, d, pad, code):
    for which in ("both", "resid", "y"):
        c = case(T, d, (BF, BF, BF, pad, 0), gate="channel", kind=LAYER, masked=0.2 if T > 1 else 0.0)
        resid, _, stats, _ = c.forward()
        kr, ky = c.kept(resid, code if which != "y" else None), c.kept(c.y, code if which != "resid" else None)
        o = c.backward(kr, ky, stats)
        c.check_backward(o, kr, ky, stats)
    c = case(T, d, (F, F, F, pad, 0), gate="token", kind=RMS)
    resid, _, stats, _ = c.forward()
    kr, ky = c.kept(resid, code), c.kept(c.y, code)
    c.check_backward(c.backward(kr, ky, stats), kr, ky, stats)


@pytest.mark.parametrize("code", [E4M3, INT8])
@pytest.mark.parametrize("T,d,pad", [(1300, 512, 0), (1300, 1000, 0), (1300, 2048, 16), (1300, 4096, 0), (300, 1001, 0), (1300, 1000, 3),
                                     (20, 4608, 0), (20, 6144, 0), (20, 6144, 3), (5, 8192, 0), (40, 16, 0), (40, 40, 8)])
def test_backward_from_8_bits_without_betas(T, d, pad, code):
    """The kernels for root-mean-square norms, by rows and width; types of stream and block that differ."""
    for layout, gate in (((BF, BF, BF, pad, 0), "none"), ((F, BF, F, pad, 0), "channel")):
        c = case(T, d, layout, gate=gate, kind=RMS, masked=0.2)
        resid, _, stats, _ = c.forward()
        kr, ky = c.kept(resid, code), c.kept(c.y, code)
        c.check_backward(c.backward(kr, ky, stats), kr, ky, stats)
        o = c.backward(resid, ky, stats)
        c.check_backward(o, resid, ky, stats)


@pytest.mark.parametrize("d", [6000, 7168, 8192])
def test_wide_rows_of_four_bytes(d):
    """Rows of which two do not fit in shared memory with everything: y and the gate are read beside it."""
    for gate, kind in (("token", LAYER), ("none", RMS), ("token", RMS)):
        c = case(310, d, (F, F, BF, 0, 0), gate=gate, kind=kind, masked=0.2)
        out = c.forward()
        c.check_forward(*out)
        c.check_backward(c.backward(out[0], c.y, out[2]), out[0], c.y, out[2])


@pytest.mark.parametrize("d", [96, 1001, 4096, 9000])
def test_outputs_left_out(d):
    """Each output by itself is what it is among all others."""
    for gate in ("channel", "token"):
        c = case(130, d, (BF, BF, F, 0, 0), gate=gate, kind=LAYER, masked=0.2)
        resid, _, stats, _ = c.forward()
        whole = c.backward(resid, c.y, stats)
        for name in whole:
            alone = c.backward(resid, c.y, stats, skip=[k for k in whole if k != name])
            assert torch.equal(alone[name], whole[name]), name


@pytest.mark.parametrize("d", [64, 1000, 1001, 4096, 8200])
def test_rows_that_are_not_finite(d):
    for gate, kind in (("none", RMS), ("channel", LAYER)):
        c = case(40, d, (F, F, F, 0, 0), gate=gate, kind=kind)
        c.y[3, 0], c.resid[5, d - 1], c.resid[7, 0], c.y[9, 1] = float("nan"), float("inf"), 3e38, -float("inf")
        resid, h, stats, st = c.forward()
        assert st.item() == 9
        bad = [3, 5, 7, 9]
        assert not resid[bad].any() and not h[bad].any() and not stats[bad].any()
        c.on[bad] = False
        st.zero_()
        c.check_forward(resid, h, stats, st)
        c.resid[bad], c.y[bad] = float("nan"), float("nan")
        o = c.backward(resid, c.y, stats)
        c.check_backward(o, resid, c.y, stats)


def test_every_token_masked_and_no_tokens():
    c = case(70, 640, (BF, BF, F, 0, 0), gate="token", kind=LAYER, masked=1.0)
    resid, h, stats, st = c.forward()
    assert st.item() == 0 and not resid.any() and not h.any() and not stats.any()
    o = c.backward(resid, c.y, stats)
    assert not any(v.any() for v in o.values() if v is not None)
    for gate in ("channel", "none"):
        c = case(1, 640, (BF, BF, F, 0, 0), gate=gate)
        resid, h, stats, _ = c.forward()
        for n in ("resid", "y", "dh", "d_resid_out"):
            setattr(c, n, getattr(c, n)[:0])
        c.T = 0
        c.on = c.on[:0]
        c.forward()
        o = c.backward(resid[:0], c.y, stats[:0])
        assert not any(o[k].any() for k in VECTORS if o[k] is not None) and (gate == "none" or not o["dgate"].any())


@pytest.mark.parametrize("d", [1024, 1000])
def test_large_means_and_constant_rows(d):
    c = case(12, d, (F, F, F, 0, 0), kind=LAYER)
    c.y += 1000.0
    c.resid += 1000.0
    out = c.forward()
    c.check_forward(*out)
    c.y.fill_(2.0)  # the norm leaves beta of it, exactly
    c.resid.fill_(0.0)
    resid, _, _, st = c.forward()
    assert st.item() == 0 and torch.equal(resid, c.beta_post.expand(12, d))


@pytest.mark.parametrize("d", [64, 1001])
def test_rows_far_apart(d):
    """Offsets beyond 32 bits: the numbers of the same rows next to each other."""
    far = Case(5, d, BF, BF, F, kind=LAYER, gate="channel", ld=600_000_000)
    near = Case(5, d, BF, BF, F, kind=LAYER, gate="channel", ld=d if d % 8 == 0 else 1008)
    a, b = far.forward(), near.forward()
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    o, p = far.backward(a[0], far.y, a[2]), near.backward(b[0], near.y, b[2])
    assert all(torch.equal(o[k], p[k]) for k in o)
    del far, a, o
    torch.cuda.empty_cache()


def test_parameters_of_any_alignment():
    for pdt in (BF, F):
        a, b = (case(200, 1024, (BF, BF, pdt, 0, 0), kind=LAYER, gate="channel") for _ in range(2))
        for name in ("gamma_post", "beta_post", "gamma_pre", "beta_pre", "gate"):
            v = torch.zeros(1027, device="cuda", dtype=pdt)[3:]
            v.copy_(getattr(a, name))
            setattr(b, name, v)
        ra, rb = a.forward(), b.forward()
        assert all(torch.equal(x, y) for x, y in zip(ra, rb))
        oa, ob = a.backward(ra[0], a.y, ra[2]), b.backward(rb[0], b.y, rb[2])
        assert all(torch.equal(oa[k], ob[k]) for k in oa)


def test_same_bits_every_time_other_stream_and_graphs():
    c = case(900, 2048, (BF, BF, BF, 0, 0), gate="channel")
    ref = c.forward()
    back = c.backward(ref[0], c.y, ref[2])
    for _ in range(4):
        again = c.backward(ref[0], c.y, ref[2])
        assert all(back[k] is None or torch.equal(back[k], again[k]) for k in back)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        out = c.forward()
        again = c.backward(out[0], c.y, out[2])
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(ref, out)) and all(back[k] is None or torch.equal(back[k], again[k]) for k in back)
    graphs = []
    for _ in range(2):  # two graphs, each with its own buffers, replayed in turn on new values
        c.forward()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = c.forward()
            o = c.backward(out[0], c.y, out[2])
        graphs.append((graph, out, o))
    c.y.copy_(c.y.flip(0))
    c.dh.mul_(-2.0)
    for graph, _, _ in graphs:
        graph.replay()
    torch.cuda.synchronize()
    want = c.forward()
    back = c.backward(want[0], c.y, want[2])
    for _, out, o in graphs:
        assert all(torch.equal(a, b) for a, b in zip(want, out)) and all(o[k] is None or torch.equal(o[k], back[k]) for k in back)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("gate", ["none", "channel", "token"])
def test_gradients_against_autograd_and_differences(kind, gate):
    """fp32 throughout: the chain of forward and backward pass against float64 autograd of the formula, and against central
    differences of the kernel's own forward pass.  The differences: outputs of magnitude 5 are off by 1e-5 or so of
    themselves, N = T d of them enter with random signs, and the error is divided by 2 eps: sqrt(N) 5e-5 / 2e-2, beside
    <grad, v> of about sqrt(N); 2 % allowed, with eps^2 terms."""
    T, d = 24, 160
    c = case(T, d, (F, F, F, 0, 0), kind=kind, gate=gate, alpha=0.8, s=0.5)
    out = c.forward()
    o = c.backward(out[0], c.y, out[2])
    names = ["resid", "y", "gamma_post", "gamma_pre"] + (["beta_post", "beta_pre"] if kind == LAYER else []) + (["gate"] if c.gate is not None else [])
    back = dict(resid="d_resid", y="dy", gate="dgate", gamma_post="dgamma_post", gamma_pre="dgamma_pre", beta_post="dbeta_post", beta_pre="dbeta_pre")
    own = {n: getattr(c, n) for n in names}
    leaves = {n: own[n].double().requires_grad_() for n in names}
    for n in names:
        setattr(c, n, leaves[n])
    r64, h64, _, _ = c.formula(leaves["resid"], leaves["y"])
    loss = (r64 * c.d_resid_out.double()).sum() + (h64 * c.dh.double()).sum()
    grads = dict(zip(names, torch.autograd.grad(loss, list(leaves.values()))))
    for n in names:
        got, want = o[back[n]].double(), grads[n]
        assert float((got - want).norm()) <= 3e-5 * float(want.norm()), n
        setattr(c, n, own[n])
    eps = 1e-2
    for n in names:
        v = torch.randn(own[n].shape, generator=c.g, device="cuda")
        losses = []
        for sign in (1.0, -1.0):
            setattr(c, n, own[n] + sign * eps * v)
            r, h, _, _ = c.forward()
            losses.append((r.double() * c.d_resid_out.double()).sum() + (h.double() * c.dh.double()).sum())
        setattr(c, n, own[n])
        got, want = float((o[back[n]].double() * v.double()).sum()), float((losses[0] - losses[1]) / (2 * eps))
        assert abs(got - want) <= 0.02 * float((o[back[n]].double() ** 2).sum().sqrt()), n


@pytest.mark.parametrize("gate", ["channel", "token"])
@pytest.mark.parametrize("d,pad", [(16, 0), (96, 0), (1001, 0), (1000, 3), (4096, 0), (5120, 0), (6144, 0), (9000, 0)])
def test_betas_without_their_gradients(d, pad, gate):
    """Root-mean-square norms with betas whose own gradients are not asked for: beta is in the gate's gradient all the same,
    with all other outputs and by itself, in rows that begin alike and in rows that do not."""
    for T, layout in ((130, (BF, BF, F, pad, 0)), (130, (F, F, BF, pad, 0)), (1300, (BF, BF, BF, pad, 0))):
        c = case(T, d, layout, gate=gate, kind=RMS, beta=True, masked=0.2, s=0.5)
        resid, _, stats, _ = c.forward()
        frozen = ("dbeta_post", "dbeta_pre")
        alike = c.y
        for y in (alike, strided(T, d, c.ld + 5, 1, c.ydt).copy_(alike)):
            c.y = y
            o = c.backward(resid, y, stats, skip=frozen)
            c.check_backward(o, resid, y, stats)
            alone = c.backward(resid, y, stats, skip=[k for k in o if k != "dgate"])
            c.check_backward(alone, resid, y, stats)


@pytest.mark.parametrize("code", [E4M3, INT8])
@pytest.mark.parametrize("T,d,kind", [(3000, 512, RMS), (3000, 4096, RMS), (1500, 5120, RMS), (3000, 2048, LAYER), (1500, 6144, LAYER)])
def test_backward_from_8_bits_same_bits_every_time(T, d, kind, code):
    """Codes that a warp copies together, over many rows to a group: each is read before the next row's come into its place."""
    c = case(T, d, (BF, BF, BF, 0, 0), gate="channel", kind=kind, masked=0.1)
    resid, _, stats, _ = c.forward()
    kr, ky = c.kept(resid, code), c.kept(c.y, code)
    first = c.backward(kr, ky, stats)
    c.check_backward(first, kr, ky, stats)
    for _ in range(10):
        again = c.backward(kr, ky, stats)
        assert all(torch.equal(first[k], again[k]) for k in first)


@pytest.mark.parametrize("code", [None, E4M3, INT8])
@pytest.mark.parametrize("d,pad", [(512, 0), (1000, 0), (1001, 0), (1000, 3), (8201, 0)])
def test_masked_rows_are_of_no_effect(d, pad, code):
    """Whatever they hold: codes and exponents of any bits, statistics and gradients that are not finite."""
    for gate, kind in (("channel", RMS), ("token", LAYER)):
        c = case(700, d, (BF, BF, BF, pad, 0), gate=gate, kind=kind, masked=0.4)
        resid, _, stats, _ = c.forward()
        kr, ky = c.kept(resid, code), c.kept(c.y, code)
        first = c.backward(kr, ky, stats)
        c.check_backward(first, kr, ky, stats)
        off = ~c.on
        for x in (kr, ky):
            if code is None:
                x[off] = float("inf")
            else:
                x[0].view(torch.uint8)[off] = 127  # NaN among e4m3 codes
                x[1][off] = 255
        stats[off] = float("nan")
        c.dh[off], c.d_resid_out[off] = -float("inf"), float("inf")
        again = c.backward(kr, ky, stats)
        assert all(torch.equal(first[k], again[k]) for k in first)


NO_BETAS = ("dbeta_post", "dbeta_pre")


@pytest.mark.parametrize("gate", ["none", "channel", "token"])
@pytest.mark.parametrize("T,d,pad", [(40, 16, 0), (1300, 256, 0), (1300, 264, 0), (1300, 512, 0), (1300, 2048, 8), (1300, 4096, 0), (700, 4104, 0),
                                     (700, 5120, 0), (330, 6144, 0), (330, 8192, 0), (1300, 1001, 0), (330, 1000, 3), (330, 3001, 0),
                                     (330, 4101, 0), (330, 6147, 0), (330, 8191, 0)])
def test_backward_of_root_mean_square_norms_alone(T, d, pad, gate):
    """No betas and no gradients of any: the kernels without the means of layer norms and the sums for betas -- two pieces to a
    thread from 1,216 rows of 257 to 4,096 columns, 640 threads above that, two pieces again above 5,120 -- by what r' and y
    are stored in, and rows that begin anywhere."""
    for k, (rdt, ydt) in enumerate(((BF, BF), (F, BF), (BF, F), (F, F))):
        c = case(T, d, (rdt, ydt, (BF, F)[k % 2], pad, 0), gate=gate, kind=RMS, masked=0.2 if k else 0.0, s=0.5, alpha=(1.0, 0.7)[k // 2])
        resid, _, stats, _ = c.forward()
        for r_code, y_code in ((None, None), (E4M3, E4M3), (INT8, INT8), (None, E4M3), (INT8, None)):
            kr, ky = c.kept(resid, r_code), c.kept(c.y, y_code)
            c.check_backward(c.backward(kr, ky, stats, skip=NO_BETAS), kr, ky, stats)


@pytest.mark.parametrize("code", [None, E4M3, INT8])
@pytest.mark.parametrize("T,d,pad", [(1300, 512, 0), (1300, 4096, 0), (330, 5120, 0), (330, 8192, 0), (330, 1001, 0), (330, 6147, 0)])
def test_root_mean_square_norms_with_parts_missing(T, d, pad, code):
    """The same without the stream's gradient, without one norm or its gradients, and each output by itself."""
    for post, pre in ((True, True), (False, True), (True, False)):
        for gate in ("none", "channel", "token"):
            c = case(T, d, (BF, BF, F, pad, 0), gate=gate, kind=RMS, post=post, pre=pre, masked=0.2)
            resid, _, stats, _ = c.forward()
            kr = c.kept(resid, code) if pre else None
            ky = c.kept(c.y, code) if post or gate != "none" else None
            whole = c.backward(kr, ky, stats, skip=NO_BETAS)
            c.check_backward(whole, kr, ky, stats)
            if pre:
                c.check_backward(c.backward(kr, ky, stats, skip=NO_BETAS, d_resid_out=None), kr, ky, stats, dro=None)
            for name in whole:
                if whole[name] is not None:
                    alone = c.backward(kr, ky, stats, skip=[k for k in whole if k != name])
                    c.check_backward(alone, kr, ky, stats)
