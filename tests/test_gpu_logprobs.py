"""Token log probabilities, entropies, top alternatives and their gradient against float64.

Tolerances.  A log probability is (z - m) - log S.  z - m is rounded once (2^-24 of itself); log S
carries the error of a sum of V terms of one sign, each off by 2^-22 at most, added up in partial sums of at
most V / 32 terms: up to 2^-22 + V / 32 * 2^-24 in the worst case, and the square root of that count in
earnest.  1e-5 + 1e-6 |lp| holds both for V up to 150,000 with a margin of 3.  Where y is all but certain both
outputs are sums of terms of one sign and good to 1e-4 of themselves.  A gradient element is a product of
p (relative error = absolute error of lp, 2e-5) with factors of the same error.
"""
import numpy as np
import pytest
import torch

import paper_2607_05804_gb300 as P

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def forward(z, V, y=None, rows=None, mask=None, n_top=0, stream=None):
    T = next((t.numel() for t in (mask, y, rows) if t is not None), z.shape[0])
    new = lambda *s: torch.full(s, 7.0, device="cuda")  # noqa: E731
    o = dict(lp=new(T) if y is not None else None, H=new(T), stats=new(T, 2),
             ids=torch.full((T, n_top), 7, dtype=torch.int32, device="cuda") if n_top else None,
             tlp=new(T, n_top) if n_top else None, status=torch.zeros(1, dtype=torch.int32, device="cuda"))
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda") if mask is not None else None
    P.turnopd_token_logprobs(z, V, rows, y, mask, n_top, o["lp"], o["H"], o["stats"], o["ids"], o["tlp"], ws, o["status"],
                             stream)
    return o


def reference(z, V, y, n_top):
    """Of rows z in float64: lp of y, H, m, log S, ids (ties: the lower id), their lp, and the whole log softmax."""
    x = z[:, :V].double()
    m = x.amax(1, keepdim=True)
    logs = (x - m).exp().sum(1, keepdim=True).log()
    lp = x - m - logs
    if y is not None:
        # y's own: -log(1 + S') from the sum over the others, which 64 bits would lose beside 1
        yy = y[:, None].long()
        others = (x - x.gather(1, yy)).exp().scatter(1, yy, 0.0).sum(1, keepdim=True)
        lp.scatter_(1, yy, torch.where(torch.isfinite(others) & (others < 1), -torch.log1p(others), lp.gather(1, yy)))
    p = lp.exp()
    H = -torch.where(p > 0, p * lp, 0.0).sum(1)
    ids = torch.sort(x + 0.0, dim=1, descending=True, stable=True).indices[:, :n_top]
    py = lp.gather(1, y[:, None].long())[:, 0] if y is not None else None
    return py, H, m[:, 0], logs[:, 0], ids, lp.gather(1, ids), lp


def close(a, b, tol):
    a, b = a.double(), b.double()
    inf = torch.isinf(b)
    assert torch.equal(a[inf], b[inf])
    err = (a - b)[~inf].abs()
    lim = (tol if torch.is_tensor(tol) else torch.full_like(b, tol))[~inf]
    assert bool((err <= lim).all()), float((err / lim).max())


def check_forward(o, z, V, y, n_top, at=None):
    py, H, m, logs, ids, tlp, _ = reference(z, V, y, n_top)
    pick = (lambda t: t) if at is None else (lambda t: t[at])
    if y is not None:
        close(pick(o["lp"]), py, 1e-5 + 1e-6 * py.abs())
        sure = py > -1e-3
        if bool(sure.any()):
            close(pick(o["lp"])[sure], py[sure], 1e-4 * py[sure].abs() + 1e-30)
            close(pick(o["H"])[sure], H[sure], 1e-4 * H[sure].abs() + 1e-30)
    close(pick(o["H"]), H, 2e-5 + 1e-6 * H)
    assert torch.equal(pick(o["stats"])[:, 0].double(), m)
    close(pick(o["stats"])[:, 1], logs, 1e-5)
    if n_top:
        assert torch.equal(pick(o["ids"]).long(), ids)
        close(pick(o["tlp"]), tlp, 1e-5 + 1e-6 * tlp.abs())


def make(n, V, dtype, seed, ld=None, offset=0, scale=3.0):
    """Rows of a strided, possibly unaligned array; one id of each row raised by 0 to 30."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    ld = V if ld is None else ld
    z = torch.full((n * ld + offset,), 1e30, device="cuda", dtype=dtype)[offset:].view(n, ld)  # gaps hold large values
    a = torch.randn((n, V), generator=g, device="cuda") * scale
    a.scatter_(1, torch.randint(V, (n, 1), generator=g, device="cuda"), 30 * torch.rand((n, 1), generator=g, device="cuda"))
    z[:, :V] = a.to(dtype)
    y = torch.argmax(z[:, :V].float() - torch.empty((n, V), device="cuda").exponential_(generator=g).log(), 1).int()
    return z, y


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("V,ld,offset,n_top", [
    (1, 1, 0, 1), (2, 3, 1, 2), (7, 7, 1, 7), (31, 40, 3, 31), (32, 32, 0, 32), (33, 33, 5, 32), (255, 256, 0, 20),
    (1000, 1000, 0, 5), (1024, 1024, 0, 0), (2049, 2049, 7, 20), (8192, 8192, 0, 32), (8193, 8200, 0, 1),
    (16385, 16385, 2, 32), (50001, 50001, 0, 10), (50304, 50304, 0, 0), (151936, 151936, 0, 20)])
def test_sizes_and_strides(dtype, V, ld, offset, n_top):
    for n in (1, 5, 70):
        z, y = make(n, V, dtype, seed=V + n, ld=ld, offset=offset)
        o = forward(z, V, y, n_top=n_top)
        assert o["status"].item() == 0
        check_forward(o, z, V, y, n_top)


@pytest.mark.parametrize("n", [2, 17, 100, 160, 310, 620, 1300])
def test_row_counts(n):
    """Every way of sharing the device out among the rows."""
    for dtype, V in ((BF, 9000), (F, 30011)):
        z, y = make(n, V, dtype, seed=n, ld=V + 1)
        o = forward(z, V, y, n_top=20)
        check_forward(o, z, V, y, 20)


@pytest.mark.parametrize("dtype", [BF, F])
def test_orders_and_ties(dtype):
    V = 40_000
    up = torch.linspace(-5, 5, V, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(3)
    rows = [up, up.flip(0), torch.zeros(V, device="cuda"), torch.full((V,), -2.5, device="cuda"),
            (torch.arange(V, device="cuda") % 2).float() - 0.5, torch.round(torch.randn(V, generator=g, device="cuda")),
            torch.where(torch.arange(V, device="cuda") % 3 == 0, -0.0, 0.0),
            (torch.arange(V, device="cuda") % 2048).float() / 256, (torch.arange(V, device="cuda") // 2048).float() / 4,
            torch.where(torch.arange(V, device="cuda") >= V - 40, 4.0, 0.0),
            torch.where(torch.arange(V, device="cuda") % 1024 == 1023, 4.0, 0.0)]
    z = torch.stack(rows).to(dtype)
    y = torch.randint(V, (z.shape[0],), generator=g, device="cuda").int()
    for n_top in (1, 20, 32):
        check_forward(forward(z, V, y, n_top=n_top), z, V, y, n_top)
    many = z.repeat(60, 1)
    check_forward(forward(many, V, y.repeat(60), n_top=32), many, V, y.repeat(60), 32)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("gone", [-float("inf"), "lowest"])
def test_forbidden_vocabulary(dtype, gone):
    """Forbidden tokens as -inf or as the type's lowest value, down to one token that is left."""
    V, low = 20_000, torch.finfo(dtype).min
    fill = low if gone == "lowest" else gone
    z, y = make(6, V, dtype, seed=9)
    for r, keep in enumerate((1, 2, 3, 19, 200, V - 1)):
        kept = torch.randperm(V, device="cuda")[:keep]
        kept[0] = y[r]
        row = torch.full((V,), fill, device="cuda", dtype=dtype)
        row[kept] = z[r, kept]
        z[r] = row
    y2 = y.clone()
    y2[2] = int((z[2] == fill).nonzero()[0])  # a forbidden token was given: log probability -inf, or the lowest value
    for yy in (y, y2):
        o = forward(z, V, yy, n_top=20)
        assert o["status"].item() == 0
        py, H, m, logs, ids, tlp, _ = reference(z, V, yy, 20)
        close(o["lp"], py, 1e-5 + 1e-6 * py.abs())
        close(o["H"], H, 2e-5 + 1e-6 * H)
        assert torch.equal(o["ids"].long(), ids)
        close(o["tlp"], tlp, 1e-5 + 1e-6 * tlp.abs())
    assert o["lp"][0].item() == 0.0 and abs(o["H"][0].item()) == 0.0


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("fill", [-1e33, -1e35, -1e37, -8e37])
@pytest.mark.parametrize("n,V", [(6, 20_000), (6, 151_936), (310, 20_000), (620, 20_000), (620, 151_936)])
def test_forbidden_vocabulary_of_any_fill(dtype, fill, n, V):
    """Forbidden tokens as any large negative number, with one CTA and with several to a row."""
    z, y = make(n, V, dtype, seed=n)
    for r in range(n):
        kept = torch.randperm(V, device="cuda")[:(1, 2, 3, 19, 200, V - 1)[r % 6]]
        kept[0] = y[r]
        row = torch.full((V,), fill, device="cuda", dtype=dtype)
        row[kept] = z[r, kept]
        z[r] = row
    y2 = y.clone()
    y2[2] = int((z[2] == z[2].min()).nonzero()[0])  # a forbidden one was given
    for yy in (y, y2):
        o = forward(z, V, yy, n_top=20)
        assert o["status"].item() == 0
        check_forward(o, z, V, yy, 20)
    gl, gh = torch.linspace(-1, 1, n, device="cuda"), torch.linspace(1, 2, n, device="cuda")
    out = torch.empty_like(z)
    P.turnopd_token_logprobs_bwd(z, V, None, y2, None, o["stats"], o["lp"], o["H"], gl, gh, out, 0, None, o["status"])
    check_grad(out, z, V, y2, gl, gh)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n", [3, 310, 620])
def test_one_logit_far_above_the_rest(dtype, n):
    V = 20_000
    for at in (0, 7, 9000, V - 1):
        z, y = make(n, V, dtype, seed=at + 1)
        z[:, at] = 1e37
        y[::2] = at
        o = forward(z, V, y, n_top=5)
        assert o["status"].item() == 0
        check_forward(o, z, V, y, 5)


def test_masks_rows_and_skipped_tokens():
    V, T = 5003, 300
    z, _ = make(40, V, BF, seed=1, ld=5008)
    g = torch.Generator(device="cuda").manual_seed(2)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    rows = torch.randint(40, (T,), generator=g, device="cuda").int()  # several tokens share a row
    y = torch.randint(V, (T,), generator=g, device="cuda").int()
    rows[mask == 0] = -5
    y[mask == 0] = V + 3
    for m in (mask, torch.zeros_like(mask), None):
        r, yy = (rows, y) if m is not None else (rows.clamp(min=0), y.clamp(max=V - 1))
        o = forward(z, V, yy, rows=r, mask=m, n_top=4)
        assert o["status"].item() == 0
        on = torch.ones(T, dtype=torch.bool, device="cuda") if m is None else m.bool()
        check_forward(o, z[r[on].long()], V, yy[on], 4, at=on)
        off = ~on
        assert (o["lp"][off] == 0).all() and (o["H"][off] == 0).all() and (o["ids"][off] == -1).all()
        assert (o["tlp"][off] == 0).all() and (o["stats"][off] == 0).all()
    # indexes out of range: reported, those tokens as if masked, the others right
    bad_r, bad_y = rows.clone(), y.clone()
    on = mask.nonzero()[:, 0]
    bad_r[on[0]], bad_r[on[1]], bad_y[on[2]], bad_y[on[3]] = 40, -1, V, -2
    for m in (mask, None):
        rr, yy = (bad_r, bad_y) if m is not None else (bad_r.clamp(max=40), bad_y)
        o = forward(z, V, yy, rows=rr, mask=m, n_top=4)
        assert o["status"].item() == 5
        assert (o["lp"][on[:4]] == 0).all() and (o["ids"][on[:4]] == -1).all()
        assert (o["stats"][on[:4], 0] == -float("inf")).all()
        rest = on[4:]
        check_forward(o, z[rr[rest].long()], V, yy[rest], 4, at=rest)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_non_finite_rows_are_reported(dtype, bad):
    V = 3001
    for col in (0, 1500, V - 1):
        for n in (3, 400):
            z, y = make(n, V, dtype, seed=col + 5)
            z[1, col] = bad
            o = forward(z, V, y, n_top=3)
            assert o["status"].item() == 9
            assert o["lp"][1] == 0 and o["H"][1] == 0 and o["stats"][1, 0] == -float("inf") and (o["ids"][1] == -1).all()
            ok = torch.arange(n, device="cuda") != 1
            check_forward(o, z[ok], V, y[ok], 3, at=ok)
        y[1] = col
        assert forward(z, V, y, n_top=3)["status"].item() == 9
    z, y = make(2, V, dtype, seed=8)
    z[0] = -float("inf")  # nothing left of a row
    o = forward(z, V, y, n_top=3)
    assert o["status"].item() == 9 and o["lp"][0] == 0
    check_forward({k: (v[1:] if v is not None and v.numel() > 1 else v) for k, v in o.items()}, z[1:], V, y[1:], 3)


def test_without_tokens_and_single_outputs():
    V = 4097
    z, y = make(9, V, BF, seed=4)
    o = forward(z, V, None, n_top=3)
    check_forward(o, z, V, None, 3)
    lp = torch.empty(9, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_token_logprobs(z, V, None, y, None, 0, lp, None, None, None, None, None, st)
    close(lp, reference(z, V, y, 1)[0], 1e-5 + 1e-6 * lp.abs().double())


def test_offsets_beyond_32_bits():
    """The last rows of an array of 2.3 G logits, read and written."""
    V, n = 151_936, 15_200
    z = torch.zeros((n, V), dtype=BF, device="cuda")
    last, y = make(3, V, BF, seed=6)
    z[-3:] = last
    rows = torch.tensor([n - 3, n - 2, n - 1], dtype=torch.int32, device="cuda")
    o = forward(z, V, y, rows=rows, n_top=5)
    check_forward(o, last, V, y, 5)
    gl = torch.ones(3, device="cuda")
    P.turnopd_token_logprobs_bwd(z, V, rows, y, None, o["stats"], o["lp"], o["H"], gl, None, z, 0, None, o["status"])
    check_grad(z[-3:], last, V, y, gl, torch.zeros(3, device="cuda"))
    assert not z[:-3].any() and o["status"].item() == 0


def test_longest_row_read_once_for_each_alternative():
    """A row of 2^31 - 1 logits whose first chunk qualifies too many: five lanes' vectors of every 32 hold 4, the others 0,
    so the sixth best of the groups is a 0.  203 tokens: one CTA takes the row."""
    V, T = 2 ** 31 - 1, 203
    z = torch.zeros(2 ** 31, dtype=BF, device="cuda")
    z.view(-1, 32, 8)[:, :5] = 4.0
    rows, mask = torch.zeros(T, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[7] = 1
    o = forward(z[:V].view(1, V), V, None, rows=rows, mask=mask, n_top=6)
    assert o["status"].item() == 0
    assert o["ids"][7].tolist() == [0, 1, 2, 3, 4, 5] and (o["ids"][mask == 0] == -1).all()
    assert o["stats"][7, 0] == 4.0


def test_same_bits_on_every_run_and_stream():
    V = 30_000
    z, y = make(333, V, BF, seed=12)
    a = forward(z, V, y, n_top=20)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        b = forward(z, V, y, n_top=20)
    s.synchronize()
    for k in a:
        assert torch.equal(a[k], b[k]), k


# ---------------------------------------------------------------- gradient

def grad64(z, V, y, gl, gh):
    py, H, _, _, _, _, lp = reference(z, V, y, 1)
    p = lp.exp()
    gl, gh = gl.double()[:, None], gh.double()[:, None]
    pl = torch.where(p > 0, p * (lp + H[:, None]), 0.0)
    yy = y[:, None].long()
    rest = p.scatter(1, yy, 0.0).sum(1, keepdim=True)
    g = (-gl * p).scatter(1, yy, gl * rest) - gh * pl
    size = (gl.abs() * p).scatter(1, yy, gl.abs() * rest) + gh.abs() * torch.where(p > 0, p * (lp.abs() + H[:, None] + 1), 0.0)
    return g, size


def check_grad(g, z, V, y, gl, gh):
    ref, size = grad64(z, V, y, gl, gh)
    tol = 1e-4 * size + 1e-30
    if g.dtype == BF:
        tol = tol + 2.0 ** -8 * ref.abs() + 1e-37
    close(g[:, :V], ref, tol)


@pytest.mark.parametrize("din,dout", [(BF, BF), (BF, F), (F, F), (F, BF)])
@pytest.mark.parametrize("V,ld,offset", [(1, 1, 0), (3, 5, 1), (8, 8, 0), (1001, 1001, 1), (1024, 1024, 0), (4097, 4104, 0),
                                         (16385, 16385, 3), (50001, 50001, 0), (151936, 151936, 0)])
def test_gradient(din, dout, V, ld, offset):
    for n in (1, 6, 50):
        z, y = make(n, V, din, seed=V + n, ld=ld, offset=offset)
        o = forward(z, V, y)
        g = torch.Generator(device="cuda").manual_seed(n)
        gl, gh = torch.randn(n, generator=g, device="cuda"), torch.randn(n, generator=g, device="cuda")
        for a, b in ((gl, gh), (gl, None), (None, gh)):
            out = torch.full((n * ld + offset,), 3.0, device="cuda", dtype=dout)[offset:].view(n, ld)
            P.turnopd_token_logprobs_bwd(z, V, None, y, None, o["stats"], o["lp"], o["H"], a, b, out, 0, None, o["status"])
            assert o["status"].item() == 0
            check_grad(out, z, V, y, a if a is not None else torch.zeros_like(gl), b if b is not None else torch.zeros_like(gh))
            if ld > V:
                assert (out[:, V:] == 3.0).all()


@pytest.mark.parametrize("dtype", [BF, F])
def test_gradient_in_place(dtype):
    V = 10_007
    z, y = make(200, V, dtype, seed=2)
    o = forward(z, V, y)
    gl = torch.linspace(-1, 1, 200, device="cuda")
    want = torch.empty_like(z)
    P.turnopd_token_logprobs_bwd(z, V, None, y, None, o["stats"], o["lp"], o["H"], gl, gl, want, 0, None, o["status"])
    P.turnopd_token_logprobs_bwd(z, V, None, y, None, o["stats"], o["lp"], o["H"], gl, gl, z, 0, None, o["status"])
    assert torch.equal(z, want)


def test_gradient_masks_and_skipped_tokens():
    V, T = 5003, 120
    z, y = make(T, V, BF, seed=3)
    g = torch.Generator(device="cuda").manual_seed(4)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    on = mask.nonzero()[:, 0]
    z[on[5], 17] = float("nan")
    z[on[6], :] = -float("inf")
    z[on[7], :4000] = -float("inf")  # forbidden tokens have no gradient
    y[on[7]] = 4500
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    o = forward(z, V, y, mask=mask)
    assert o["status"].item() == 9
    o["status"].zero_()
    gl, gh = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    for flags in (0, P.TURNOPD_ZERO_MASKED_GRAD):
        out = torch.full_like(z, 3.0)
        P.turnopd_token_logprobs_bwd(z, V, None, y, mask, o["stats"], o["lp"], o["H"], gl, gh, out, flags, ws, o["status"])
        assert o["status"].item() == 0
        rest = torch.cat([on[:5], on[7:]])
        check_grad(out[rest], z[rest], V, y[rest], gl[rest], gh[rest])
        assert (out[on[7], :4000] == 0).all()
        assert not out[on[5]].any() and not out[on[6]].any()
        off = (mask == 0).nonzero()[:, 0]
        assert (out[off] == (0.0 if flags else 3.0)).all()
    # compact rows, one of them out of range: nothing of it is written
    rows = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    rows[on] = torch.arange(on.numel(), device="cuda").int()
    rows[on[2]] = on.numel()
    zc = z[on].contiguous()
    out = torch.full_like(zc, 3.0)
    P.turnopd_token_logprobs_bwd(zc, V, rows, y, mask, o["stats"], o["lp"], o["H"], gl, gh, out, 0, ws, o["status"])
    assert o["status"].item() == 5 and (out[2] == 3.0).all()
    check_grad(out[8:], zc[8:], V, y[on[8:]], gl[on[8:]], gh[on[8:]])


@pytest.mark.parametrize("T", [60, 3000])
def test_masked_tokens_that_point_at_supervised_rows(T):
    """A token -> row map with 0 for masked tokens: row 0 keeps its supervised token's gradient."""
    V = 3000
    g = torch.Generator(device="cuda").manual_seed(T)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    on = mask.nonzero()[:, 0]
    z, y_row = make(on.numel(), V, F, seed=T)
    rows = torch.zeros(T, dtype=torch.int32, device="cuda")
    rows[on] = torch.arange(on.numel(), device="cuda").int()
    y = torch.zeros(T, dtype=torch.int32, device="cuda")
    y[on] = y_row
    o = forward(z, V, y, rows=rows, mask=mask)
    gl = torch.randn(T, generator=g, device="cuda")
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    out = torch.full_like(z, 3.0)
    P.turnopd_token_logprobs_bwd(z, V, rows, y, mask, o["stats"], o["lp"], o["H"], gl, None, out, P.TURNOPD_ZERO_MASKED_GRAD,
                                 ws, o["status"])
    check_grad(out, z, V, y[on], gl[on], torch.zeros_like(gl[on]))


def test_gradient_against_differences():
    """Along random directions, against central differences of the float64 objective."""
    V, n = 777, 8
    z, y = make(n, V, F, seed=5, scale=1.0)
    z.clamp_(max=6.0)
    o = forward(z, V, y)
    gl, gh = torch.linspace(-1, 2, n, device="cuda"), torch.linspace(1, -0.5, n, device="cuda")
    out = torch.empty_like(z)
    P.turnopd_token_logprobs_bwd(z, V, None, y, None, o["stats"], o["lp"], o["H"], gl, gh, out, 0, None, o["status"])

    def f(x):
        lp = torch.log_softmax(x, 1)
        return (gl.double() * lp.gather(1, y[:, None].long())[:, 0] - gh.double() * (lp.exp() * lp).sum(1)).sum()

    u = torch.randn((5, n, V), generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.float64)
    for k in range(5):
        h = 1e-4
        diff = (f(z.double() + h * u[k]) - f(z.double() - h * u[k])) / (2 * h)
        got = (out.double() * u[k]).sum()
        size = (out.double() * u[k]).abs().sum()
        assert abs(diff - got) <= 1e-4 * size + 1e-6


@pytest.mark.parametrize("T", [5, 3000])
def test_compact_layout_without_rows(T):
    """No token is supervised, so no row of logits is there: every output is a masked token's.  A token that is supervised
    all the same has no row to name."""
    V = 1000
    z, grad = torch.empty((0, V), device="cuda"), torch.empty((0, V), device="cuda")
    rows, y = torch.full((T,), -1, dtype=torch.int32, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    gl = torch.ones(T, device="cuda")
    for on in (None, 3):
        mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
        if on is not None:
            mask[on], rows[on] = 1, 0
        o = forward(z, V, y, rows=rows, mask=mask, n_top=4)
        assert o["status"].item() == (0 if on is None else 5)
        assert not o["lp"].any() and not o["H"].any() and (o["ids"] == -1).all() and not o["tlp"].any()
        want = torch.zeros((T, 2), device="cuda")
        if on is not None:
            want[on, 0] = -float("inf")
        assert torch.equal(o["stats"], want)
        for flags in (0, P.TURNOPD_ZERO_MASKED_GRAD):
            o["status"].zero_()
            P.turnopd_token_logprobs_bwd(z, V, rows, y, mask, o["stats"], o["lp"], o["H"], gl, gl, grad, flags, ws, o["status"])
            assert o["status"].item() == (0 if on is None else 5)
    with pytest.raises(P.TurnopdError):  # a row to each token: none may be missing
        forward(z, V, y, n_top=4)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("n_top", [0, 7])
@pytest.mark.parametrize("on", [0, 1, 2, 700, 1063, 1064, 1065, 2999, 3000])
def test_lists_of_few_and_of_many_rows(on, n_top, dtype):
    """Tokens enough for a list of the supervised ones, with none, few, as many as CTAs and all of them on it."""
    V, T = 1003, 3000
    z, y = make(T, V, dtype, seed=on, ld=1008)
    mask = torch.zeros(T, dtype=torch.uint8, device="cuda")
    mask[torch.randperm(T, device="cuda", generator=torch.Generator(device="cuda").manual_seed(on))[:on]] = 1
    at, off = mask.nonzero()[:, 0], (mask == 0).nonzero()[:, 0]
    z[off] = float("nan")
    o = forward(z, V, y, mask=mask, n_top=n_top)
    assert o["status"].item() == 0
    if on:
        check_forward(o, z[at], V, y[at], n_top, at=at)
    assert not o["lp"][off].any() and not o["H"][off].any() and not o["stats"][off].any()
    if n_top:
        assert (o["ids"][off] == -1).all() and not o["tlp"][off].any()
    gl = torch.linspace(-1, 1, T, device="cuda")
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    for flags, left in ((0, 3.0), (P.TURNOPD_ZERO_MASKED_GRAD, 0.0)):
        out = torch.full_like(z, 3.0)
        P.turnopd_token_logprobs_bwd(z, V, None, y, mask, o["stats"], o["lp"], o["H"], gl, gl, out, flags, ws, o["status"])
        assert o["status"].item() == 0 and (out[off, :V] == left).all() and (out[:, V:] == 3.0).all()
        if on:
            check_grad(out[at], z[at], V, y[at], gl[at], gl[at])


@pytest.mark.parametrize("T", [300, 3000])
@pytest.mark.parametrize("dtype", [BF, F])
def test_tokens_that_are_not_on_the_list(T, dtype):
    """Masked tokens and indexes out of range where the kernels look at the mask themselves (300 tokens) and where the
    supervised ones are listed (3,000): every output of such a token, and its gradient left alone."""
    V, R = 2003, 50
    z, _ = make(R, V, dtype, seed=T, ld=2008)
    g = torch.Generator(device="cuda").manual_seed(T)
    mask = (torch.rand(T, generator=g, device="cuda") < 0.5).to(torch.uint8)
    rows, y = (torch.randint(n, (T,), generator=g, device="cuda").int() for n in (R, V))
    off, on = (mask == 0).nonzero()[:, 0], mask.nonzero()[:, 0]
    rows[off], y[off] = -7, V + 9
    bad = on[[0, 1, 2, 3, -1]]
    rows[bad[0]], rows[bad[1]], y[bad[2]], y[bad[3]], rows[bad[4]] = R, -1, V, -2, 2 ** 31 - 1
    o = forward(z, V, y, rows=rows, mask=mask, n_top=4)
    assert o["status"].item() == 5
    good = on[4:-1]
    check_forward(o, z[rows[good].long()], V, y[good], 4, at=good)
    for at, m in ((off, 0.0), (bad, -float("inf"))):
        assert not o["lp"][at].any() and not o["H"][at].any() and (o["ids"][at] == -1).all() and not o["tlp"][at].any()
        assert (o["stats"][at, 0] == m).all() and (o["stats"][at, 1] == 0).all()
    # a row to each supervised token; one token has no row, one an id out of range, and their rows are left alone
    rows = torch.full((T,), -1, dtype=torch.int32, device="cuda")
    rows[on] = torch.arange(on.numel(), device="cuda").int()
    zc, yc = make(on.numel(), V, dtype, seed=T + 1, ld=2008)
    y[on] = yc
    rows[bad[1]], y[bad[4]] = on.numel(), V
    rest = torch.ones(on.numel(), dtype=torch.bool, device="cuda")
    rest[[1, -1]] = False
    o = forward(zc, V, y, rows=rows, mask=mask)
    assert o["status"].item() == 5
    gl, gh = torch.randn(T, generator=g, device="cuda"), torch.randn(T, generator=g, device="cuda")
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(T), dtype=torch.uint8, device="cuda")
    for flags in (0, P.TURNOPD_ZERO_MASKED_GRAD):
        out = torch.full_like(zc, 3.0)
        o["status"].zero_()
        P.turnopd_token_logprobs_bwd(zc, V, rows, y, mask, o["stats"], o["lp"], o["H"], gl, gh, out, flags, ws, o["status"])
        assert o["status"].item() == 5 and (out[~rest] == 3.0).all() and (out[:, V:] == 3.0).all()
        check_grad(out[rest], zc[rest], V, y[on[rest]], gl[on[rest]], gh[on[rest]])


def test_ties_across_clusters_of_eight():
    """70,000 bf16 columns and few rows: eight CTAs to a row, ties within and across their slices."""
    V = 70_000
    i = torch.arange(V, device="cuda")
    rows = [torch.zeros(V, device="cuda"), (i % 2).float(), (i // 8750).float(), -(i // 8750).float(), (i % 8750 == 0).float(),
            (i >= V - 20).float(), torch.where(i % 8192 == 8191, 1.0, -1.0), torch.linspace(-4, 4, V, device="cuda")]
    z = torch.stack(rows).to(BF)
    y = torch.arange(len(rows), device="cuda").int() * 9001
    for n_top in (1, 9, 32):
        check_forward(forward(z, V, y, n_top=n_top), z, V, y, n_top)


@pytest.mark.parametrize("n,V,masked", [(3, 151_936, False), (700, 5003, False), (3000, 1003, True)])
def test_in_a_cuda_graph(n, V, masked):
    """Both calls captured and replayed on new logits give the bits of the calls outside."""
    z, y = make(n, V, BF, seed=n)
    z2, _ = make(n, V, BF, seed=n + 1)
    mask = (torch.arange(n, device="cuda") % 3 != 0).to(torch.uint8) if masked else None
    gl = torch.linspace(-1, 1, n, device="cuda")
    new = lambda *s: torch.zeros(s, device="cuda")  # noqa: E731
    lp, H, stats, tlp, out = new(n), new(n), new(n, 2), new(n, 5), torch.zeros_like(z)
    ids, st = torch.zeros((n, 5), dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(P.turnopd_token_logprobs_workspace_bytes(n), dtype=torch.uint8, device="cuda")

    def both(stream=None):
        P.turnopd_token_logprobs(z, V, None, y, mask, 5, lp, H, stats, ids, tlp, ws, st, stream)
        P.turnopd_token_logprobs_bwd(z, V, None, y, mask, stats, lp, H, gl, gl, out, P.TURNOPD_ZERO_MASKED_GRAD if masked else 0,
                                     ws, st, stream)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    z.copy_(z2)
    for _ in range(2):
        graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (lp, H, stats, ids, tlp, out)]
    both()
    assert st.item() == 0 and all(torch.equal(a, b) for a, b in zip(got, (lp, H, stats, ids, tlp, out)))
    check_forward(forward(z, V, y, n_top=5), z, V, y, 5)


def test_nothing_to_do():
    z = torch.zeros((0, 64), device="cuda")
    o = forward(z, 64)
    assert o["H"].numel() == 0 and o["status"].item() == 0


def test_refusals():
    z, y = make(4, 100, F, seed=1)
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    lp, H, stats = torch.zeros(4, device="cuda"), torch.zeros(4, device="cuda"), torch.zeros((4, 2), device="cuda")
    f = lambda **k: P.turnopd_token_logprobs(**{**dict(  # noqa: E731
        logits=z, vocab=100, row_of_token=None, token_ids=y, loss_mask=None, n_top=0, logprob_out=lp, entropy_out=H,
        stats_out=stats, top_ids_out=None, top_logprob_out=None, workspace=None, dev_status=st), **k})
    for k in (dict(vocab=101), dict(logits=z.half()), dict(logits=z.t()), dict(token_ids=y.long()), dict(logprob_out=lp[:3]),
              dict(logprob_out=lp.double()), dict(logits=z.cpu())):
        with pytest.raises(ValueError):
            f(**k)
    top = dict(top_ids_out=torch.zeros((4, 33), dtype=torch.int32, device="cuda"), top_logprob_out=torch.zeros((4, 33), device="cuda"))
    for k, code in ((dict(n_top=33, **top), 2), (dict(n_top=1), 1), (dict(token_ids=None), 1), (dict(vocab=0), 2),
                    (dict(loss_mask=torch.ones(4, dtype=torch.uint8, device="cuda")), 10)):
        with pytest.raises((P.TurnopdError, ValueError)) as e:
            f(**k)
        assert not isinstance(e.value, P.TurnopdError) or e.value.code == code
    g = torch.empty((4, 100), device="cuda")
    with pytest.raises(ValueError):
        P.turnopd_token_logprobs_bwd(z, 100, None, y, None, stats, lp, H, lp, None, g[:, :99], 0, None, st)
    with pytest.raises(P.TurnopdError):
        P.turnopd_token_logprobs_bwd(z, 100, None, y, None, stats, lp, H, None, None, g, 0, None, st)
    assert st.item() == 0
