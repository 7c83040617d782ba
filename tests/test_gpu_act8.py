"""Activations in 8 bits: codes, exponents and loaded values against the definition in float64.  Scaling by a power of two is
exact, so everything has to be equal bit for bit; the loss is at most half a step of the code."""
import math

import pytest
import torch

import paper_2607_05804_gb300 as P

pytestmark = pytest.mark.gpu
BF, F = torch.bfloat16, torch.float32
E4M3, INT8 = torch.float8_e4m3fn, torch.int8
TOP = {E4M3: 448.0, INT8: 127.0}


def strided(T, d, ld, offset, dtype, fill):
    return torch.full((T * ld + offset,), fill, device="cuda", dtype=dtype)[offset:].view(T, ld)[:, :d]


def codes_buffer(T, d, ld, offset, dtype):
    return torch.full((T * ld + offset,), 77, device="cuda", dtype=torch.uint8).view(dtype)[offset:].view(T, ld)[:, :d]


def reference(x, code):
    """Exponent bytes and values, a group at a time, in float64 on the CPU."""
    x = x.double().cpu()
    T, d = x.shape
    n = (d + 31) // 32
    exps, out = torch.zeros((T, n), dtype=torch.uint8), torch.zeros_like(x)
    for g in range(n):
        v = x[:, 32 * g:32 * g + 32]
        for i in range(T):
            most = float(v[i].abs().max())
            if not math.isfinite(most):
                exps[i, g] = 255
                out[i, 32 * g:32 * g + 32] = math.nan
                continue
            k = -126
            if most > 0:
                k = math.frexp(most)[1] - 10
                while most > TOP[code] * 2.0 ** k:
                    k += 1
                k = max(k, -126)
            exps[i, g] = k + 127
            w = v[i] / 2.0 ** k
            step = torch.ones_like(w)
            if code is E4M3:
                step = 2.0 ** (torch.frexp(w.abs().clamp(min=2.0 ** -6)).exponent - 4).double()
            out[i, 32 * g:32 * g + 32] = torch.round(w / step) * step * 2.0 ** k
    return exps, out


def store(x, code, mask=None, ldc=None, offset=0):
    T, d = x.shape
    q = codes_buffer(T, d, ldc or d, offset, code)
    exps = torch.full((T, (d + 31) // 32), 33, dtype=torch.uint8, device="cuda")
    st = torch.zeros(1, dtype=torch.int32, device="cuda")
    P.turnopd_act8_store(x, mask, q, exps, st)
    return q, exps, st


def same(a, b):
    return torch.equal(torch.nan_to_num(a.double().cpu(), nan=1e300), torch.nan_to_num(b.double().cpu(), nan=1e300))


@pytest.mark.parametrize("code", [E4M3, INT8])
@pytest.mark.parametrize("T,d", [(1, 1), (2, 7), (3, 31), (2, 32), (5, 33), (1, 256), (3, 257), (7, 1001), (40, 520), (2, 4096)])
def test_round_trip(T, d, code):
    g = torch.Generator(device="cuda").manual_seed(T * d)
    for dt, ld, off in ((BF, d, 0), (F, d, 0), (BF, d + 8 - d % 8, 0), (F, d + 3, 1), (BF, d + 1, 1)):
        x = strided(T, d, ld, off, dt, 9.0)
        # magnitudes from far below the code's smallest step to the largest of a group
        x.copy_(torch.randn((T, d), generator=g, device="cuda") * torch.exp2(torch.randint(-14, 15, (T, d), generator=g, device="cuda").float()))
        x[0, 0] = 0.0
        exps64, out64 = reference(x, code)
        for ldc, offc in ((d, 0), (d + 8 - d % 8, 8), (d + 5, 3)):
            q, exps, st = store(x, code, ldc=ldc, offset=offc)
            assert st.item() == 0 and torch.equal(exps.cpu(), exps64)
            for odt in (BF, F):
                out = strided(T, d, ld, off, odt, 5.0)
                P.turnopd_act8_load(q, exps, out)
                assert same(out, out64)
            if ldc > d:  # what stands between the rows is left alone
                whole = torch.as_strided(q.view(torch.uint8), (T, ldc), (ldc, 1)) if T > 1 else None
                assert whole is None or bool((whole[:-1, d:] == 77).all())


@pytest.mark.parametrize("code", [E4M3, INT8])
def test_ties_edges_and_extremes(code):
    """Ties to even, group maxima next to a power of two times the largest code, subnormals, zeros, the type's ends."""
    top = TOP[code]
    rows = [[top, top * (1 + 2.0 ** -20), top * (1 - 2.0 ** -20)], [1.0625, 1.1875, 448.0], [0.5, 1.5, 2.5, 127.0],
            [2.0 ** -149, 2.0 ** -140, -2.0 ** -126], [0.0, -0.0], [2.0 ** -10 * 448, 2.0 ** -11 * 448, 448.0, 1.5 * 2.0 ** -9],
            [3.4e38, -3.4028234663852886e38], [1e-37, -3e-38], [top * 2.0 ** 119, 1.0], [2.0 ** 127, 2.0 ** 120]]
    x = torch.zeros((len(rows), 32), device="cuda")
    for i, r in enumerate(rows):
        x[i, :len(r)] = torch.tensor(r, dtype=torch.float64).float()
    q, exps, st = store(x, code)
    exps64, out64 = reference(x, code)
    out = torch.empty_like(x)
    P.turnopd_act8_load(q, exps, out)
    assert st.item() == 0 and torch.equal(exps.cpu(), exps64) and same(out, out64.clamp(-3.4028234663852886e38, 3.4028234663852886e38))
    b = torch.tensor([[-3.3895313892515355e38] * 32], device="cuda").to(BF)  # the lowest bf16 stays finite
    q, exps, st = store(b, code)
    out = torch.empty_like(b)
    P.turnopd_act8_load(q, exps, out)
    assert st.item() == 0 and bool(torch.isfinite(out).all()) and bool(((out / b - 1).abs() <= 2.0 ** -4).all())


@pytest.mark.parametrize("code", [E4M3, INT8])
@pytest.mark.parametrize("ld", [96, 97])
def test_masks_and_non_finite_groups(code, ld):
    T, d = 20, 96
    x = strided(T, d, ld, 0, F, 0.0)
    x.copy_(torch.randn((T, d), device="cuda"))
    mask = torch.ones(T, dtype=torch.uint8, device="cuda")
    mask[3:6] = 0
    x[4] = math.nan  # not read
    q, exps, st = store(x, code, mask=mask, ldc=ld)
    assert st.item() == 0 and not exps[3:6].any() and not q[3:6].float().any()
    out = torch.empty((T, d), device="cuda")
    P.turnopd_act8_load(q, exps, out)
    assert not out[3:6].any()
    x[7, 40], x[8, 0], x[9, 95] = math.nan, math.inf, -math.inf
    q, exps, st = store(x, code, mask=mask, ldc=ld)
    P.turnopd_act8_load(q, exps, out)
    assert st.item() == 9
    bad = torch.zeros((T, 3), dtype=torch.bool, device="cuda")
    bad[7, 1] = bad[8, 0] = bad[9, 2] = True
    assert torch.equal(exps == 255, bad) and torch.equal(torch.isnan(out), bad.repeat_interleave(32, 1))
    zero = torch.zeros_like(mask)
    q, exps, st = store(x, code, mask=zero, ldc=ld)
    assert st.item() == 0 and not exps.any() and not q.float().any()
    # no tokens at all
    P.turnopd_act8_store(x[:0], None, q[:0], exps[:0], st)
    P.turnopd_act8_load(q[:0], exps[:0], out[:0])


def test_many_rows_other_stream_and_graph():
    """More work than the grid has warps; another stream; captured and replayed with other values."""
    T, d = 5000, 776
    x = torch.randn((T, d), device="cuda").to(BF)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    q, exps = torch.empty((T, d), dtype=E4M3, device="cuda"), torch.empty((T, (d + 31) // 32), dtype=torch.uint8, device="cuda")
    st, out = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.empty_like(x)
    with torch.cuda.stream(s):
        P.turnopd_act8_store(x, None, q, exps, st)
    P.turnopd_act8_load(q, exps, out, stream=s)
    s.synchronize()
    k = exps.int().repeat_interleave(32, 1)[:, :d] - 127
    assert torch.equal(out.float(), torch.ldexp(q.float(), k))
    assert bool(((out.double() - x.double()).abs() <= x.double().abs() * 2.0 ** -4 + torch.ldexp(torch.full_like(x, 2.0 ** -10, dtype=F), k).double()).all())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.turnopd_act8_store(x, None, q, exps, st)
        P.turnopd_act8_load(q, exps, out)
    first = out.clone()
    x.mul_(-3.0)
    graph.replay()
    torch.cuda.synchronize()
    got = out.clone()
    P.turnopd_act8_store(x, None, q, exps, st)
    P.turnopd_act8_load(q, exps, out)
    assert torch.equal(got, out) and not torch.equal(got, first) and st.item() == 0


@pytest.mark.parametrize("d", [64, 1001])
def test_rows_far_apart(d):
    """Offsets beyond 32 bits in values and codes."""
    ld, T = 600_000_000, 5
    x = strided(T, d, ld, 0, BF, 0.0)
    x.copy_(torch.randn((T, d), device="cuda"))
    q, exps, st = store(x, INT8, ldc=1_200_000_000)
    q2, exps2, _ = store(x.contiguous(), INT8)
    out = strided(T, d, ld, 0, BF, 0.0)
    P.turnopd_act8_load(q, exps, out)
    assert st.item() == 0 and torch.equal(q, q2) and torch.equal(exps, exps2)
    near = torch.empty((T, d), device="cuda", dtype=BF)
    P.turnopd_act8_load(q2, exps2, near)
    assert torch.equal(out, near)
    del x, q, out
    torch.cuda.empty_cache()


@pytest.mark.parametrize("d", [32, 33])
def test_values_below_the_smallest_of_bf16(d):
    """e4m3 codes reach down to 2^-135, bf16 to 2^-133: what lies between is rounded to the nearest one, ties to even."""
    n = torch.arange(-16, d - 16, dtype=torch.float64)
    x = (n * 2.0 ** -135).float()[None].repeat(2, 1).cuda()  # codes up to sixteen of the smallest steps: exact
    for code in (E4M3, INT8):
        q, exps, st = store(x, code)
        wide, out = torch.empty_like(x), torch.empty((2, d), device="cuda", dtype=BF)
        P.turnopd_act8_load(q, exps, wide)
        P.turnopd_act8_load(q, exps, out)
        assert st.item() == 0 and bool((exps == 1).all())
        exact = (n if code is E4M3 else torch.zeros_like(n)) * 2.0 ** -135
        assert same(wide[0], exact)
        assert same(out[0], torch.round(exact * 2.0 ** 133) * 2.0 ** -133) and torch.equal(out[0], out[1])
