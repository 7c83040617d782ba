"""Embedding lookup and its gradient against float64.

Tolerances.  The lookup is one fp32 product, rounded to the output's type: 2^-24 and half a step of that type.  The gradient
sums the n rows of an id in fp32 in some fixed order, each addition rounded to 2^-24 of a partial sum that is at most the sum
of magnitudes S: (n + 2) 2^-24 |scale| S with the product and an old value's addition, and half a step of the output's type.
"""
import pytest
import torch

import paper_2607_05804_gb300 as P

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32


def strided(rows, d, ld, offset, dtype, fill=3.0):
    return torch.full((rows * ld + offset,), fill, device="cuda", dtype=dtype)[offset:].view(rows, ld)[:, :d]


def half_step(t):
    return torch.finfo(t).eps / 2


def within(a, b, tol):
    err = (a.double() - b).abs()
    assert bool(torch.isfinite(a.double()).all()) and bool((err <= tol).all()), float((err - tol).max())


def backward(dout, ids, V, scale, wdt, mask=None, dw=None, flags=0, ldw=None, offset=0, stream=None):
    T, d = dout.shape
    if dw is None:
        dw = strided(V, d, ldw or d, offset, wdt)
    ws = torch.empty(P.turnopd_embedding_bwd_workspace_bytes(T, d, V), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_embedding_bwd(dout, ids, mask, scale, dw, flags, ws, st, stream)
    return dw, st


def check_backward(dw, dout, ids, V, scale, on=None, old=None):
    d = dout.shape[1]
    on = torch.ones_like(ids, dtype=torch.bool) if on is None else on
    i = ids[on].long()
    ref = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, i, dout[on].double()) * scale
    size = torch.zeros((V, d), dtype=torch.float64, device="cuda").index_add_(0, i, dout[on].double().abs()) * abs(scale)
    n = torch.bincount(i, minlength=V)[:, None]
    tol = (n + 2) * 2.0 ** -24 * size
    if old is not None:
        ref, tol = ref + old.double(), tol + 2.0 ** -23 * old.double().abs()
    within(dw, ref, tol + half_step(dw.dtype) * ref.abs() + (1e-38 if dw.dtype is BF else 1e-44))
    untouched = n[:, 0] == 0
    assert torch.equal(dw[untouched], torch.zeros_like(dw[untouched]) if old is None else old[untouched])


@pytest.mark.parametrize("T,d,V", [(1, 1, 1), (1, 4096, 151_936), (5, 7, 3), (64, 1024, 1000), (300, 1001, 77), (3, 8200, 11),
                                   (20_000, 64, 513)])
def test_lookup(T, d, V):
    g = torch.Generator(device="cuda").manual_seed(T + d)
    ids = torch.randint(V, (T,), generator=g, device="cuda").int()
    for wdt, odt, ld, off, scale in ((BF, BF, d, 0, 1.0), (BF, F, d, 0, 3.3), (F, BF, d + 8 - d % 8, 0, d ** 0.5),
                                     (F, F, d + 3, 1, -0.7), (BF, BF, d + 1, 1, 64.0)):
        w, out = strided(V, d, ld, off, wdt, 0.0), strided(T, d, ld, off, odt)
        w.copy_(torch.randn((V, d), generator=g, device="cuda"))
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        P.turnopd_embedding_fwd(w, ids, None, scale, out, st)
        s = float(torch.tensor(scale, dtype=F))
        ref = w[ids.long()].double() * s
        within(out, ref, (2.0 ** -24 + (half_step(BF) if odt is BF else 0.0)) * ref.abs() + 1e-40)
        assert st.item() == 0
        if scale == 1.0 and wdt is odt:
            assert torch.equal(out, w[ids.long()])


def test_lookup_masks_and_ids_out_of_range():
    for d, ld in ((96, 96), (97, 97)):
        w, out = torch.randn((50, ld), device="cuda")[:, :d], torch.full((9, ld + 2), 3.0, device="cuda")
        ids = torch.tensor([0, 49, -1, 50, 7, 2**31 - 1, -2**31, 3, 3], dtype=torch.int32, device="cuda")
        mask = torch.tensor([1, 1, 0, 0, 0, 0, 0, 1, 1], dtype=torch.uint8, device="cuda")
        st = torch.zeros(1, dtype=torch.int32, device="cuda")
        P.turnopd_embedding_fwd(w, ids, mask, 1.0, out[:, :d], st)  # ids of masked tokens are not looked at
        assert st.item() == 0 and torch.equal(out[[0, 1, 7, 8], :d], w[[0, 49, 3, 3]]) and not out[2:7, :d].any()
        assert (out[:, d:] == 3.0).all()
        P.turnopd_embedding_fwd(w, ids, None, 1.0, out[:, :d], st)
        assert st.item() == 5 and torch.equal(out[[0, 1, 4], :d], w[[0, 49, 7]]) and not out[[2, 3, 5, 6], :d].any()


@pytest.mark.parametrize("T,d,V", [(1, 1, 1), (1, 4096, 3000), (7, 5, 4), (8, 64, 2), (9, 33, 40), (256, 256, 1024), (1000, 1001, 31),
                                   (1025, 72, 100_003), (3000, 2056, 200), (9000, 16, 5), (40_000, 24, 262_150)])
def test_gradient(T, d, V):
    g = torch.Generator(device="cuda").manual_seed(T + V)
    # frequencies from 1 to much of the batch
    ids = (V ** torch.rand(T, generator=g, device="cuda", dtype=torch.float64)).long().clamp(1, V).sub_(1).int()
    for gdt, wdt, ld, off, scale in ((BF, BF, d, 0, 1.0), (F, F, d, 0, 8.0), (BF, F, d + 8 - d % 8, 0, 0.3), (F, BF, d + 3, 1, 1.0),
                                     (BF, BF, d + 1, 1, 2.0)):
        dout = strided(T, d, ld, off, gdt, 0.0)
        dout.copy_(torch.randn((T, d), generator=g, device="cuda"))
        s = float(torch.tensor(scale, dtype=F))
        dw, st = backward(dout, ids, V, scale, wdt, ldw=ld, offset=off)
        assert st.item() == 0
        check_backward(dw, dout, ids, V, s)
        old = strided(V, d, ld, off, wdt)
        old.copy_(torch.randn((V, d), generator=g, device="cuda"))
        dw = strided(V, d, ld, off, wdt)
        dw.copy_(old)
        dw, st = backward(dout, ids, V, scale, wdt, dw=dw, flags=P.TURNOPD_ACCUMULATE_GRAD)
        assert st.item() == 0
        check_backward(dw, dout, ids, V, s, old=old)


@pytest.mark.parametrize("T", [1, 8, 9, 64, 1024, 1025, 8191, 8192, 8193, 70_001])
def test_one_id_for_every_token_and_one_id_each(T):
    """A run over every tile, and no run at all; whole numbers, so the sums are exact."""
    d = 40
    dout = torch.randint(-3, 4, (T, d), device="cuda").float()
    ids = torch.full((T,), 2, dtype=torch.int32, device="cuda")
    dw, st = backward(dout, ids, 5, 1.0, F)
    assert st.item() == 0 and torch.equal(dw[2], dout.sum(0)) and not dw[[0, 1, 3, 4]].any()
    ids = torch.randperm(T + 3, device="cuda")[:T].int()
    dw, _ = backward(dout, ids, T + 3, 1.0, F)
    assert torch.equal(dw[ids.long()], dout) and int((dw != 0).any(1).sum()) == int((dout != 0).any(1).sum())


def test_runs_that_end_at_tile_ends():
    """Runs of 1 to 40 tokens over 8-token tiles: every place where a run can begin and end in a tile."""
    lengths = torch.tensor([(7 * k) % 40 + 1 for k in range(120)], device="cuda")
    ids = torch.repeat_interleave(torch.arange(120, device="cuda"), lengths).int()
    ids = ids[torch.randperm(ids.numel(), device="cuda")]
    dout = torch.randint(-9, 10, (ids.numel(), 33), device="cuda").float()
    dw, _ = backward(dout, ids, 120, 1.0, F)
    assert torch.equal(dw, torch.zeros((120, 33), device="cuda").index_add_(0, ids.long(), dout))


@pytest.mark.parametrize("T,d,V,pad,wdt", [(1, 520, 70_001, 0, F), (3000, 520, 70_001, 0, F), (20_000, 1001, 70_033, 0, BF),
                                           (3000, 1000, 70_000, 3, BF), (9000, 2056, 33_001, 8, BF)])
def test_tables_beyond_what_is_zeroed_beside_the_sort(T, d, V, pad, wdt):
    """The rest of the zeros goes out beside the sums: absent rows only, whatever the table held."""
    dout = torch.randint(-3, 4, (T, d), device="cuda").to(BF)
    ids = (V ** torch.rand(T, device="cuda", dtype=torch.float64)).long().clamp(1, V).sub_(1)
    ids = torch.randperm(V, device="cuda")[ids].int()
    dw, st = backward(dout, ids, V, 1.0, wdt, ldw=d + pad)
    assert st.item() == 0
    check_backward(dw, dout, ids, V, 1.0)


def test_gradient_masks_and_ids_out_of_range():
    T, d, V = 500, 48, 60
    dout = torch.randn((T, d), device="cuda")
    ids = torch.randint(V, (T,), device="cuda").int()
    mask = (torch.rand(T, device="cuda") < 0.5).to(torch.uint8)
    dout[mask == 0] = float("nan")
    ids[(mask == 0).nonzero()[:3, 0]] = -5
    dw, st = backward(dout, ids, V, 1.0, F, mask=mask)
    assert st.item() == 0
    check_backward(dw, dout, ids, V, 1.0, on=mask.bool())
    on = mask.bool()
    bad = on.nonzero()[:4, 0]
    ids[bad] = torch.tensor([-1, V, 2**31 - 1, -2**31], dtype=torch.int32, device="cuda")
    on[bad] = False
    dw, st = backward(dout, ids, V, 1.0, F, mask=mask)
    assert st.item() == 5
    check_backward(dw, dout, ids, V, 1.0, on=on)
    dw, st = backward(dout, ids, V, 1.0, BF, mask=torch.zeros_like(mask))  # nothing takes part
    assert st.item() == 0 and not dw.any()
    dw, st = backward(dout[:0], ids[:0], V, 1.0, F)  # no tokens
    assert st.item() == 0 and not dw.any()
    old = torch.randn((V, d), device="cuda")
    dw, st = backward(dout, ids, V, 1.0, F, mask=torch.zeros_like(mask), dw=old.clone(), flags=P.TURNOPD_ACCUMULATE_GRAD)
    assert torch.equal(dw, old)


@pytest.mark.parametrize("T,d,V", [(700, 520, 3001), (6000, 520, 3001), (20_000, 520, 70_001)])
def test_same_bits_every_time_and_in_a_graph(T, d, V):
    dout = torch.randn((T, d), device="cuda")
    ids = (V ** torch.rand(T, device="cuda")).long().clamp(1, V).sub_(1).int()
    first, _ = backward(dout, ids, V, 1.0, F)
    for _ in range(5):
        assert torch.equal(backward(dout, ids, V, 1.0, F)[0], first)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other, _ = backward(dout, ids, V, 1.0, F)
    s.synchronize()
    assert torch.equal(other, first)
    ws = [torch.empty(P.turnopd_embedding_bwd_workspace_bytes(T, d, V), dtype=torch.uint8, device="cuda") for _ in range(2)]
    st, dw, out = torch.zeros(1, dtype=torch.int32, device="cuda"), [torch.empty_like(first) for _ in range(2)], torch.empty_like(dout)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for k in range(2):
            P.turnopd_embedding_bwd(dout, ids, None, 1.0, dw[k], 0, ws[k], st)
        P.turnopd_embedding_fwd(dw[0], ids, None, 1.0, out, st)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dw[0], first) and torch.equal(dw[1], first) and torch.equal(out, first[ids.long()])
    ids.copy_(ids.flip(0))
    graph.replay()
    torch.cuda.synchronize()
    check_backward(dw[0], dout, ids, V, 1.0)
    assert st.item() == 0


def test_gradient_against_differences():
    """L = sum c out is linear in w: its difference along a direction is <dw, v>."""
    T, d, V = 300, 40, 25
    ids = torch.randint(V, (T,), device="cuda").int()
    c, w, v = torch.randn((T, d), device="cuda"), torch.randn((V, d), device="cuda"), torch.randn((V, d), device="cuda")
    st, outs = torch.zeros(1, dtype=torch.int32, device="cuda"), []
    for sign in (1.0, -1.0):
        out = torch.empty((T, d), device="cuda")
        P.turnopd_embedding_fwd(w + sign * v, ids, None, 2.5, out, st)
        outs.append((out.double() * c.double()).sum())
    dw, _ = backward(c, ids, V, 2.5, F)
    got, want = (dw.double() * v.double()).sum(), (outs[0] - outs[1]) / 2
    assert abs(got - want) <= 1e-5 * (dw.double().abs() * (v.double().abs() + w.double().abs())).sum()


@pytest.mark.parametrize("d", [64, 1001])
def test_rows_far_apart(d):
    """Offsets beyond 32 bits in the table, its gradient and the tokens' rows."""
    ld, n = 600_000_000, 5
    ids = torch.tensor([4, 0, 4, 2, 1], dtype=torch.int32, device="cuda")
    w, out = strided(n, d, ld, 0, BF), strided(n, d, ld, 0, BF)
    w.copy_(torch.randn((n, d), device="cuda"))
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_embedding_fwd(w, ids, None, 1.0, out, st)
    assert torch.equal(out, w[ids.long()])
    dw, _ = backward(out, ids, n, 1.0, BF, dw=w)  # over the table, which is no longer needed
    check_backward(dw, out, ids, n, 1.0)
    del w, out, dw
    torch.cuda.empty_cache()


def test_one_workspace_for_batches_of_any_size():
    """A workspace made for the largest batch, filled with other bits, serves every smaller one."""
    d, V = 4096, 300
    ws = torch.empty(P.turnopd_embedding_bwd_workspace_bytes(9000, d, V), dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    for T in (8176, 8192, 9000, 40, 1):
        ids = torch.randint(V, (T,), device="cuda").int()
        dout = torch.randint(-3, 4, (T, d), device="cuda").to(BF)
        dw = torch.full((V, d), 3.0, device="cuda")
        ws.fill_(255)
        P.turnopd_embedding_bwd(dout, ids, None, 1.0, dw, 0, ws, st)
        assert st.item() == 0
        check_backward(dw, dout, ids, V, 1.0)


@pytest.mark.parametrize("T,V", [(8193, 70_001), (20_000, 513), (70_001, 262_150)])
def test_sort_by_clusters_of_a_portable_size(T, V):
    """Where a cluster of sixteen CTAs cannot be placed eight sort the tokens: the same bits."""
    d = 40
    dout = torch.randn((T, d), device="cuda")
    ids = (V ** torch.rand(T, device="cuda", dtype=torch.float64)).long().clamp(1, V).sub_(1).int()
    mask = (torch.rand(T, device="cuda") < 0.8).to(torch.uint8)
    ref, _ = backward(dout, ids, V, 1.0, F, mask=mask)
    got, st = backward(dout, ids, V, 1.0, F, mask=mask, flags=P.TURNOPD_FORCE_PORTABLE)
    assert st.item() == 0 and torch.equal(got, ref)
    check_backward(got, dout, ids, V, 1.0, on=mask.bool())
    old = torch.randn((V, d), device="cuda")
    both = [backward(dout, ids, V, 1.0, F, mask=mask, dw=old.clone(), flags=P.TURNOPD_ACCUMULATE_GRAD | f)[0] for f in (0, P.TURNOPD_FORCE_PORTABLE)]
    assert torch.equal(*both)
