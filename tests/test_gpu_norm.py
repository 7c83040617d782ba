"""Layer norm, root-mean-square norm and their backward pass against float64.

Tolerances.  mu is a sum of d terms with an error of a few 2^-24 of mean |x| (partial sums of at most d / 32
terms, added up in a tree), and x - mu is rounded once, so xh is off by 1e-5 (1 + |xh| + |mu| r) at most, and y by
that times |gamma|; its rounding to bf16 adds 2^-9 of it (2^-8 allowed).  dx is a sum of three terms, each good to
2e-5 of the sums of magnitudes it is made of; dgamma and dbeta to 2e-5 of the sum of their terms' magnitudes.
"""
import pytest
import torch

import paper_2607_05804_gb300 as P

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
LAYER, RMS = P.TURNOPD_LAYER_NORM, P.TURNOPD_RMS_NORM


def strided(T, d, ld, offset, dtype, fill=1e30):
    return torch.full((T * ld + offset,), fill, device="cuda", dtype=dtype)[offset:].view(T, ld)[:, :d]


def make(T, d, dtype, seed, ld=None, offset=0, shift=0.5):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = strided(T, d, ld or d, offset, dtype)
    scale = torch.where(torch.rand(d, generator=g, device="cuda") < 0.02, 25.0, 1.0)
    x.copy_(torch.randn((T, d), generator=g, device="cuda") * scale + shift)
    gamma = 1 + 0.3 * torch.randn(d, generator=g, device="cuda")
    beta = 0.2 * torch.randn(d, generator=g, device="cuda")
    return x, gamma, beta, g


def forward(x, gamma, beta, kind, ydt, mask=None, eps=1e-6, ldy=None, offset=0, stats=True, stream=None):
    T, d = x.shape
    y = strided(T, d, ldy or d, offset, ydt, fill=3.0)
    mean, rstd = (torch.full((T,), 7.0, device="cuda") for _ in range(2))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_norm_fwd(x, gamma, beta, mask, kind, eps, y, mean if stats else None, rstd if stats else None, st, stream)
    return y, mean, rstd, st


def parts64(x, kind, eps):
    x = x.double()
    mu = x.mean(1, keepdim=True) if kind == LAYER else torch.zeros_like(x[:, :1])
    r = 1 / torch.sqrt(((x - mu) ** 2).mean(1, keepdim=True) + eps)
    return mu, r, (x - mu) * r


def within(a, b, tol):
    err = (a.double() - b).abs()
    assert bool(torch.isfinite(a.double()).all()) and bool((err <= tol).all()), float((err / tol).max())


def check_forward(y, mean, rstd, x, gamma, beta, kind, eps=1e-6):
    mu, r, xh = parts64(x, kind, eps)
    g = gamma.double()
    ref = xh * g + (beta.double() if beta is not None else 0.0)
    tol = 1e-5 * (1 + xh.abs() + mu.abs() * r) * g.abs() + 1e-6 * ref.abs() + 1e-30
    if y.dtype == BF:
        tol = tol + 2.0 ** -8 * ref.abs() + 1e-37
    within(y, ref, tol)
    if mean is not None:
        within(mean, mu[:, 0], 1e-5 * x.double().abs().mean(1) + 1e-30)
        within(rstd, r[:, 0], 1e-5 * r[:, 0] * (1 + mu[:, 0].abs() * r[:, 0]))


SHAPES = [(1, 1), (3, 2), (5, 7), (2, 8), (4, 31), (3, 127), (9, 128), (70, 255), (5, 1000), (33, 1001), (400, 1024),
          (3, 2048), (2, 4095), (1, 4096), (310, 4096), (7, 5120), (3, 8192), (2, 12000), (2, 20001), (1, 65536)]


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("T,d", SHAPES)
def test_forward(T, d, kind):
    for xdt, ydt, pdt, ld, off in ((BF, BF, BF, d, 0), (F, BF, F, d, 0), (BF, F, F, d + 3, 1), (F, F, BF, d + 8, 0),
                                   (BF, BF, F, d + 8, 8)):
        x, gamma, beta, _ = make(T, d, xdt, seed=d + T, ld=ld, offset=off)
        gamma, beta = gamma.to(pdt), beta.to(pdt)
        y, mean, rstd, st = forward(x, gamma, beta, kind, ydt, ldy=ld, offset=off)
        assert st.item() == 0
        check_forward(y, mean, rstd, x, gamma, beta, kind)
        y2, _, _, _ = forward(x, gamma, None, kind, ydt, stats=False)
        check_forward(y2, None, None, x, gamma, None, kind)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("d", [63, 511, 1001, 1537, 2047, 2601, 4100, 5119, 7003, 8191])
def test_forward_many_rows(d, kind):
    """Rows enough that as few threads as hold a row take it: every such split, with rows of any alignment and a mask."""
    T = 1300
    for xdt, ydt, ld, off in ((BF, BF, d, 0), (BF, F, d + 8 - d % 8, 0), (F, BF, d + 1, 1), (F, F, d, 0)):
        x, gamma, beta, g = make(T, d, xdt, seed=d, ld=ld, offset=off)
        mask = (torch.rand(T, generator=g, device="cuda") < 0.6).to(torch.uint8)
        x[mask == 0] = float("nan")  # masked rows are not read
        y, mean, rstd, st = forward(x, gamma, beta, kind, ydt, mask=mask, ldy=ld, offset=off)
        assert st.item() == 0
        on = mask.bool()
        check_forward(y[on], mean[on], rstd[on], x[on], gamma, beta, kind)
        assert not y[~on].any() and not mean[~on].any() and not rstd[~on].any()


def test_parameters_of_any_alignment():
    T, d = 20, 1024
    x, gamma, beta, _ = make(T, d, BF, seed=1)
    for pdt in (BF, F):
        ga, be = torch.zeros(d + 1, device="cuda", dtype=pdt), torch.zeros(d + 3, device="cuda", dtype=pdt)
        ga, be = ga[1:], be[3:]
        ga.copy_(gamma), be.copy_(beta)
        y, mean, rstd, _ = forward(x, ga, be, LAYER, BF)
        check_forward(y, mean, rstd, x, ga, be, LAYER)


def test_large_means_and_constant_rows():
    x, gamma, beta, _ = make(12, 4096, F, seed=3, shift=1000.0)
    y, mean, rstd, _ = forward(x, gamma, beta, LAYER, F)
    check_forward(y, mean, rstd, x, gamma, beta, LAYER)
    x = torch.full((3, 1024), 2.0, device="cuda")
    x[1] = 0.0
    gamma, beta = torch.ones(1024, device="cuda"), torch.full((1024,), 0.25, device="cuda")
    y, mean, rstd, st = forward(x, gamma, beta, LAYER, F, eps=1e-5)
    assert st.item() == 0 and (y == 0.25).all()  # nothing is left of a constant row but beta
    # without eps such a row has no deviation to divide by
    y, mean, rstd, st = forward(x, gamma, beta, LAYER, F, eps=0.0)
    assert st.item() == 9 and not y.any() and not rstd.any()


@pytest.mark.parametrize("d", [8, 100, 1000, 1001, 1024, 2049, 4095, 4096, 5120, 6400, 8191, 9000])
@pytest.mark.parametrize("T", [3, 1300])
def test_constant_rows_are_beta(T, d):
    """The sum of a row of equal whole numbers is exact below 2^24, and so is its d-th part: nothing is left of such a row,
    in any column, but beta."""
    for xdt, ld, off in ((BF, d, 0), (F, d, 0), (BF, d + 3, 1), (F, d + 1, 1)):
        x, gamma, beta, _ = make(T, d, xdt, seed=d, ld=ld, offset=off)
        value = torch.tensor([700.0, 1296.0, -1016.0], device="cuda").repeat(T // 3 + 1)[:T]
        x.copy_(value[:, None].expand(T, d))
        y, mean, rstd, st = forward(x, gamma, beta, LAYER, F, eps=1e-6)
        assert st.item() == 0 and torch.equal(mean, value) and torch.equal(y, beta.expand(T, d))


@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_masks_and_non_finite_rows(kind):
    T, d = 150, 1000
    x, gamma, beta, g = make(T, d, BF, seed=4, ld=1003)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    x[mask == 0] = float("nan")  # masked rows are not read
    on, off = mask.nonzero()[:, 0], (mask == 0).nonzero()[:, 0]
    y, mean, rstd, st = forward(x, gamma, beta, kind, F, mask=mask, ldy=1003)
    assert st.item() == 0 and not y[off].any() and not mean[off].any() and not rstd[off].any()
    check_forward(y[on], mean[on], rstd[on], x[on], gamma, beta, kind)
    x[on[3], 999], x[on[4], 0], x[on[5], 500] = float("nan"), float("inf"), -float("inf")
    y, mean, rstd, st = forward(x, gamma, beta, kind, F, mask=mask)
    assert st.item() == 9 and not y[on[3:6]].any() and not rstd[on[3:6]].any()
    rest = torch.cat([on[:3], on[6:]])
    check_forward(y[rest], mean[rest], rstd[rest], x[rest], gamma, beta, kind)
    dy = torch.randn((T, d), generator=g, device="cuda")
    dy[off] = float("nan")
    dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, F, mask=mask)
    assert not dx[off].any() and not dx[on[3:6]].any()
    check_backward(dx[rest], dg, db, x[rest], gamma, kind, dy[rest])
    none = torch.zeros_like(mask)
    y, mean, rstd, st = forward(x, gamma, beta, kind, F, mask=none)
    assert st.item() == 0 and not y.any()
    dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, F, mask=none)
    assert not dx.any() and not dg.any() and not db.any()


# ---------------------------------------------------------------- backward

def backward(x, gamma, kind, mean, rstd, dy, dxdt, mask=None, ldx=None, offset=0, want=(True, True, True), stream=None):
    T, d = x.shape
    dx = strided(T, d, ldx or d, offset, dxdt, fill=3.0) if want[0] else None
    dg, db = (torch.full((d,), 3.0, device="cuda") if w else None for w in want[1:])
    ws = torch.full((max(P.turnopd_norm_bwd_workspace_bytes(T, d), 256),), 0x7f, dtype=torch.uint8, device="cuda")
    P.turnopd_norm_bwd(x, gamma, mask, kind, mean if kind == LAYER else None, rstd, dy, dx, dg, db, ws, stream)
    return dx, dg, db


def check_backward(dx, dg, db, x, gamma, kind, dy, eps=1e-6):
    mu, r, xh = parts64(x, kind, eps)
    dy = dy.double()
    g = dy * gamma.double()
    m1, m2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    slack = 1 + mu.abs() * r
    if dx is not None:
        ref = r * (g - (m1 if kind == LAYER else 0.0) - xh * m2)
        tol = 2e-5 * slack * r * (g.abs() + g.abs().mean(1, keepdim=True) + (1 + xh.abs()) * (g * xh).abs().mean(1, keepdim=True)) + 1e-30
        if dx.dtype == BF:
            tol = tol + 2.0 ** -8 * ref.abs() + 1e-37
        within(dx, ref, tol)
    if dg is not None:
        within(dg, (dy * xh).sum(0), 2e-5 * (dy.abs() * (xh.abs() + slack)).sum(0) + 1e-30)
    if db is not None:
        within(db, dy.sum(0), 2e-5 * dy.abs().sum(0) + 1e-30)


@pytest.mark.parametrize("kind", [LAYER, RMS])
@pytest.mark.parametrize("T,d", SHAPES + [(2000, 64), (700, 1001), (1500, 4096)])
def test_backward(T, d, kind):
    for xdt, dydt, dxdt, pdt, ld, off in ((BF, F, BF, BF, d, 0), (F, F, F, F, d, 0), (BF, BF, BF, F, d + 3, 1),
                                          (F, BF, F, BF, d + 8, 0), (BF, F, F, F, d + 8, 8), (BF, BF, BF, BF, d, 0)):
        x, gamma, _, g = make(T, d, xdt, seed=d + T, ld=ld, offset=off)
        gamma = gamma.to(pdt)
        dy = strided(T, d, ld, off, dydt)
        dy.copy_(torch.randn((T, d), generator=g, device="cuda") * 0.01)
        _, mean, rstd, _ = forward(x, gamma, None, kind, F)
        dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, dxdt, ldx=ld, offset=off)
        check_backward(dx, dg, db, x, gamma, kind, dy)


@pytest.mark.parametrize("d,pads", [(1001, (0, 0, 0)), (1001, (3, 0, 5)), (2048, (0, 3, 0)), (4100, (1, 1, 1)), (7000, (0, 2, 0)),
                                    (320, (8, 0, 16)), (1024, (0, 0, 0))])
@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_many_masked_rows(d, pads, kind):
    """Rows enough for a list of the supervised ones, where the three arrays' rows begin alike and where they do not."""
    T = 5000
    x, gamma, _, g = make(T, d, BF, seed=d, ld=d + pads[0])
    dy = strided(T, d, d + pads[1], 0, F)
    dy.copy_(torch.randn((T, d), generator=g, device="cuda"))
    mask = (torch.rand(T, generator=g, device="cuda") < 0.4).to(torch.uint8)
    on, off = mask.nonzero()[:, 0], (mask == 0).nonzero()[:, 0]
    x[off], dy[off] = float("nan"), float("nan")
    y, mean, rstd, st = forward(x, gamma, None, kind, BF, mask=mask)
    assert st.item() == 0 and not y[off].any()
    check_forward(y[on], mean[on], rstd[on], x[on], gamma, None, kind)
    dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, BF, mask=mask, ldx=d + pads[2])
    assert not dx[off].any()
    check_backward(dx[on], dg, db, x[on], gamma, kind, dy[on])


def test_single_outputs_and_same_bits():
    T, d = 900, 2048
    x, gamma, _, g = make(T, d, BF, seed=6)
    dy = torch.randn((T, d), generator=g, device="cuda")
    _, mean, rstd, _ = forward(x, gamma, None, LAYER, BF)
    full = backward(x, gamma, LAYER, mean, rstd, dy, BF)
    check_backward(*full, x, gamma, LAYER, dy)
    for want in ((True, False, False), (False, True, False), (False, False, True), (False, True, True)):
        for got, ref, w in zip(backward(x, gamma, LAYER, mean, rstd, dy, BF, want=want), full, want):
            assert (got is None) if not w else torch.equal(got, ref)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = backward(x, gamma, LAYER, mean, rstd, dy, BF)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(full, again))


@pytest.mark.parametrize("T,d,pad", [(4400, 4096, 0), (4400, 4096, 8), (4300, 4100, 4), (2200, 8192, 0), (70_000, 256, 0),
                                     (4000, 4096, 0)])
@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_listed_rows_at_boundaries(T, d, pad, kind):
    """Elements enough for a list of the supervised rows, whose rows begin at 16-byte boundaries; the last has too few."""
    x, gamma, _, g = make(T, d, BF, seed=d, ld=d + pad)
    dy = strided(T, d, d + pad, 0, F)
    dy.copy_(torch.randn((T, d), generator=g, device="cuda"))
    mask = (torch.rand(T, generator=g, device="cuda") < 0.3).to(torch.uint8)
    on = mask.bool()
    x[~on] = float("nan")
    dy[~on] = float("nan")
    x[7], mask[7] = float("inf"), 1  # a row that the forward call reports, treated as masked
    on[7] = False
    _, mean, rstd, st = forward(x, gamma, None, kind, F, mask=mask)
    assert st.item() == 9
    dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, BF, mask=mask, ldx=d + pad)
    assert not dx[~on].any()
    check_backward(dx[on], dg, db, x[on], gamma, kind, dy[on])


@pytest.mark.parametrize("xdt,dydt", [(BF, F), (F, F), (F, BF), (BF, BF)])
@pytest.mark.parametrize("T,d", [(4400, 4096), (4300, 4100), (70_000, 256)])
@pytest.mark.parametrize("on", [0, 1, 303, 304, 305, 2433, -1])
def test_lists_of_few_and_of_many_rows(T, d, on, xdt, dydt):
    """Elements enough for a list of the supervised rows, with none, few, as many as blocks or groups and all of them on it."""
    x, gamma, _, g = make(T, d, xdt, seed=on + 2, ld=d + -d % 8)
    dy = strided(T, d, d + -d % 8, 0, dydt)
    dy.copy_(torch.randn((T, d), generator=g, device="cuda"))
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[torch.randperm(T, generator=g, device="cuda")[:on if on >= 0 else T]] = 1
    on_, off = mask.nonzero()[:, 0], mask == 0
    x[off], dy[off] = float("nan"), float("nan")
    _, mean, rstd, st = forward(x, gamma, None, LAYER, F, mask=mask)
    assert st.item() == 0
    dx, dg, db = backward(x, gamma, LAYER, mean, rstd, dy, xdt, mask=mask, ldx=d + -d % 8)
    assert not dx[off].any()
    if on_.numel():
        check_backward(dx[on_], dg, db, x[on_], gamma, LAYER, dy[on_])
    else:
        assert not dg.any() and not db.any()


@pytest.mark.parametrize("kind", [LAYER, RMS])
def test_gradient_against_differences(kind):
    """Along random directions of x, gamma and beta, against central differences of the float64 objective."""
    T, d, eps = 5, 333, 1e-5
    x, gamma, beta, g = make(T, d, F, seed=8)
    dy = torch.randn((T, d), generator=g, device="cuda")
    _, mean, rstd, _ = forward(x, gamma, beta, kind, F, eps=eps)
    dx, dg, db = backward(x, gamma, kind, mean, rstd, dy, F)

    def f(x, gamma, beta):
        return (dy.double() * (parts64(x, kind, eps)[2] * gamma + beta)).sum()

    base = [t.double() for t in (x, gamma, beta)]
    for k, grad in enumerate((dx, dg, db)):
        u = torch.randn(base[k].shape, generator=g, device="cuda", dtype=torch.float64)
        h = 1e-5
        hi, lo = ([b + s * h * u if j == k else b for j, b in enumerate(base)] for s in (1, -1))
        diff = (f(*hi) - f(*lo)) / (2 * h)
        terms = grad.double() * u
        assert abs(diff - terms.sum()) <= 1e-4 * terms.abs().sum() + 1e-6


def test_offsets_beyond_32_bits():
    T, d, ld = 3, 64, 1_200_000_000
    buf = torch.zeros(2 * ld + d, dtype=BF, device="cuda")
    x = torch.as_strided(buf, (T, d), (ld, 1))
    x.copy_(torch.randn((T, d), device="cuda"))
    out = torch.zeros(2 * ld + d, dtype=BF, device="cuda")
    y = torch.as_strided(out, (T, d), (ld, 1))
    gamma = torch.ones(d, device="cuda")
    mean, rstd, st = torch.zeros(T, device="cuda"), torch.zeros(T, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_norm_fwd(x, gamma, None, None, LAYER, 1e-6, y, mean, rstd, st)
    check_forward(y, mean, rstd, x, gamma, None, LAYER)
    dy = torch.randn((T, d), device="cuda")
    ws = torch.empty(P.turnopd_norm_bwd_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")
    dg, db = torch.zeros(d, device="cuda"), torch.zeros(d, device="cuda")
    P.turnopd_norm_bwd(x, gamma, None, LAYER, mean, rstd, dy, y, dg, db, ws)
    check_backward(y, dg, db, x, gamma, LAYER, dy)


def test_host_threads_with_rows_of_different_lengths():
    """Two host threads on streams of their own, with rows of lengths that one kernel takes with different amounts of
    shared memory: each call gets what it asks for."""
    import threading

    failed = []

    def work(d, stream, calls):
        x, gamma, beta, g = make(40, d, BF, seed=d)
        dy = torch.randn((40, d), generator=g, device="cuda")
        y, dx = torch.empty_like(x), torch.empty_like(x)
        mean, rstd = torch.empty(40, device="cuda"), torch.empty(40, device="cuda")
        dg, db, st = torch.empty(d, device="cuda"), torch.empty(d, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
        ws = torch.empty(P.turnopd_norm_bwd_workspace_bytes(40, d), dtype=torch.uint8, device="cuda")
        torch.cuda.synchronize()
        start.wait()
        try:
            for _ in range(calls):
                P.turnopd_norm_fwd(x, gamma, beta, None, LAYER, 1e-6, y, mean, rstd, st, stream)
                P.turnopd_norm_bwd(x, gamma, None, LAYER, mean, rstd, dy, dx, dg, db, ws, stream)
            stream.synchronize()
            check_forward(y, mean, rstd, x, gamma, beta, LAYER)
            check_backward(dx, dg, db, x, gamma, LAYER, dy)
        except Exception as e:  # noqa: BLE001
            failed.append((d, repr(e)))

    for lengths in ((8192, 6400), (5120, 4608)):
        start = threading.Barrier(len(lengths))
        threads = [threading.Thread(target=work, args=(d, torch.cuda.Stream(), 4000)) for d in lengths]
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    assert not failed, failed


@pytest.mark.parametrize("xdt,d", [(BF, 512), (BF, 1024), (BF, 2048), (BF, 4096), (BF, 6144), (BF, 8192), (F, 256), (F, 512),
                                   (F, 1024), (F, 1536), (F, 2048), (F, 4096), (F, 8192)])
@pytest.mark.parametrize("pad", [0, 1])
def test_rows_that_fill_every_thread(xdt, d, pad):
    """Widths whose pieces are exactly the threads' number of them, with rows few and many."""
    for T in (5, 1300):
        x, gamma, beta, _ = make(T, d, xdt, seed=d, ld=d + pad)
        for kind in (LAYER, RMS):
            y, mean, rstd, st = forward(x, gamma, beta, kind, BF, ldy=d + pad)
            assert st.item() == 0
            check_forward(y, mean, rstd, x, gamma, beta, kind)


@pytest.mark.parametrize("T,d,masked", [(3, 4096, False), (600, 1001, True), (4400, 4096, True)])
def test_in_a_cuda_graph(T, d, masked):
    """Both calls captured and replayed on new hidden states give the bits of the calls outside."""
    x, gamma, beta, g = make(T, d, BF, seed=T)
    x2 = make(T, d, BF, seed=T + 1)[0]
    dy = torch.randn((T, d), generator=g, device="cuda")
    mask = (torch.arange(T, device="cuda") % 3 != 0).to(torch.uint8) if masked else None
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    mean, rstd, dg, db = (torch.zeros(n, device="cuda") for n in (T, T, d, d))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.turnopd_norm_bwd_workspace_bytes(T, d), dtype=torch.uint8, device="cuda")

    def both():
        P.turnopd_norm_fwd(x, gamma, beta, mask, LAYER, 1e-6, y, mean, rstd, st)
        P.turnopd_norm_bwd(x, gamma, mask, LAYER, mean, rstd, dy, dx, dg, db, ws)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    x.copy_(x2)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (y, mean, rstd, dx, dg, db)]
    both()
    assert st.item() == 0 and all(torch.equal(a, b) for a, b in zip(got, (y, mean, rstd, dx, dg, db)))
    on = mask.bool() if masked else torch.ones(T, dtype=torch.bool, device="cuda")
    check_forward(y[on], mean[on], rstd[on], x[on], gamma, beta, LAYER)
    check_backward(dx[on], dg, db, x[on], gamma, LAYER, dy[on])


def test_nothing_to_do():
    x = torch.zeros((0, 64), device="cuda")
    gamma = torch.ones(64, device="cuda")
    _, _, _, st = forward(x, gamma, None, LAYER, BF)
    assert st.item() == 0
    none = torch.zeros(0, device="cuda")
    _, dg, db = backward(x, gamma, LAYER, none, none, x, BF)
    assert not dg.any() and not db.any()


def test_refusals():
    x, gamma, beta, _ = make(4, 64, BF, seed=1)
    y, st = torch.empty_like(x), torch.zeros(1, dtype=torch.int32, device="cuda")
    f = lambda **k: P.turnopd_norm_fwd(**{**dict(  # noqa: E731
        x=x, gamma=gamma, beta=beta, loss_mask=None, kind=LAYER, eps=1e-6, y_out=y, mean_out=None, rstd_out=None,
        dev_status=st), **k})
    for k in (dict(x=x.half()), dict(x=x.t()), dict(y_out=y[:3]), dict(gamma=gamma[:63]), dict(beta=beta.to(BF)),
              dict(gamma=gamma.half(), beta=None), dict(loss_mask=torch.ones(3, dtype=torch.uint8, device="cuda")),
              dict(rstd_out=torch.empty(3, device="cuda")), dict(x=x.cpu())):
        with pytest.raises(ValueError):
            f(**k)
    for k, code in ((dict(kind=2), 6), (dict(eps=-1.0), 2)):
        with pytest.raises(P.TurnopdError) as e:
            f(**k)
        assert e.value.code == code
    rstd = torch.ones(4, device="cuda")
    with pytest.raises(P.TurnopdError):  # the layer norm needs the means
        P.turnopd_norm_bwd(x, gamma, None, LAYER, None, rstd, x, y, None, None, None)
    with pytest.raises(P.TurnopdError):  # sums need a workspace
        P.turnopd_norm_bwd(x, gamma, None, RMS, None, rstd, x, None, gamma.clone(), None, None)
    assert st.item() == 0
