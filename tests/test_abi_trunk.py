"""Host-side argument checks of the embedding, the norms around a block and the 8-bit activations (they return before any
CUDA call)."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every call below fails validation first, or has nothing to do
ODD = ctypes.c_void_p(0x10001)
NULL, SHAPE, UNSUPPORTED, WORKSPACE = 1, 2, 6, 10
INF = float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05804_gb300 import build as B

    B.build()
    import paper_2607_05804_gb300 as P

    return P.load()


def test_embedding_host_validation(lib):
    def fwd(w=FAKE, wdt=1, ldw=64, V=100, ids=FAKE, T=4, d=64, scale=1.0, out=FAKE, odt=1, ldo=64, status=FAKE):
        return lib.turnopd_embedding_fwd(w, wdt, ldw, V, ids, None, T, d, scale, out, odt, ldo, status, None)

    assert fwd(w=None) == NULL and fwd(ids=None) == NULL and fwd(out=None) == NULL and fwd(status=None) == NULL
    assert fwd(wdt=2) == UNSUPPORTED and fwd(odt=3) == UNSUPPORTED
    assert fwd(ldw=63) == SHAPE and fwd(ldo=63) == SHAPE and fwd(d=0) == SHAPE and fwd(T=-1) == SHAPE and fwd(T=2**31) == SHAPE
    assert fwd(V=0) == SHAPE and fwd(V=2**31) == SHAPE and fwd(scale=INF) == SHAPE and fwd(scale=1e39) == SHAPE
    assert fwd(w=ODD) == SHAPE and fwd(out=ODD) == SHAPE and fwd(ids=ODD) == SHAPE
    assert fwd(T=0, w=None, ids=None, out=None) == 0

    need = lib.turnopd_embedding_bwd_workspace_bytes(4, 64, 100)
    assert need > 0 and lib.turnopd_embedding_bwd_workspace_bytes(0, 64, 100) > 0
    assert lib.turnopd_embedding_bwd_workspace_bytes(-1, 64, 100) == 0 == lib.turnopd_embedding_bwd_workspace_bytes(4, 0, 100)
    assert lib.turnopd_embedding_bwd_workspace_bytes(4, 64, 0) == 0

    def bwd(g=FAKE, gdt=1, ldg=64, ids=FAKE, T=4, d=64, scale=1.0, dw=FAKE, wdt=0, ldw=64, V=100, flags=0, ws=FAKE, wsb=need,
            status=FAKE):
        return lib.turnopd_embedding_bwd(g, gdt, ldg, ids, None, T, d, scale, dw, wdt, ldw, V, flags, ws, wsb, status, None)

    assert bwd(g=None) == NULL and bwd(ids=None) == NULL and bwd(dw=None) == NULL and bwd(status=None) == NULL
    assert bwd(gdt=2) == UNSUPPORTED and bwd(wdt=4) == UNSUPPORTED and bwd(flags=1) == UNSUPPORTED and bwd(flags=6) == UNSUPPORTED
    assert bwd(ldg=63) == SHAPE and bwd(ldw=63) == SHAPE and bwd(V=0) == SHAPE and bwd(scale=float("nan")) == SHAPE
    assert bwd(dw=ODD) == SHAPE and bwd(g=ODD) == SHAPE
    assert bwd(ws=None) == WORKSPACE and bwd(wsb=need - 1) == WORKSPACE and bwd(ws=ctypes.c_void_p(0x10010)) == WORKSPACE
    assert bwd(T=0, g=None, ids=None, flags=2) == 0  # nothing to add


def test_block_norm_host_validation(lib):
    def fwd(resid=FAKE, rdt=1, ldr=64, y=FAKE, ydt=1, ldy=64, gp=FAKE, bp=None, gate=None, ldg=0, g=FAKE, b=None, pdt=1, T=4,
            d=64, kind=1, eps=1e-6, alpha=1.0, s=1.0, out=ctypes.c_void_p(0x20000), ldro=64, h=FAKE, ldh=64, stats=FAKE,
            status=FAKE):
        return lib.turnopd_block_norm_fwd(resid, rdt, ldr, y, ydt, ldy, gp, bp, gate, ldg, g, b, pdt, None, T, d, kind, eps,
                                          alpha, s, out, ldro, h, ldh, stats, status, None)

    assert fwd(resid=None) == NULL and fwd(y=None) == NULL and fwd(out=None) == NULL and fwd(h=None) == NULL
    assert fwd(status=None) == NULL
    assert fwd(rdt=2) == UNSUPPORTED and fwd(ydt=3) == UNSUPPORTED and fwd(pdt=9) == UNSUPPORTED and fwd(kind=2) == UNSUPPORTED
    assert fwd(gp=None, bp=FAKE) == UNSUPPORTED and fwd(g=None, b=FAKE, h=None) == UNSUPPORTED and fwd(g=None) == UNSUPPORTED
    assert fwd(out=FAKE, ldro=72) == UNSUPPORTED  # in place needs one stride
    assert fwd(ldr=63) == SHAPE and fwd(ldy=63) == SHAPE and fwd(ldro=63) == SHAPE and fwd(ldh=63) == SHAPE
    assert fwd(gate=FAKE, ldg=63) == SHAPE and fwd(gate=ODD) == SHAPE and fwd(stats=ctypes.c_void_p(0x10008)) == SHAPE
    assert fwd(eps=-1.0) == SHAPE and fwd(eps=INF) == SHAPE and fwd(alpha=INF) == SHAPE and fwd(s=float("nan")) == SHAPE
    assert fwd(d=0) == SHAPE and fwd(T=-1) == SHAPE and fwd(resid=ODD) == SHAPE and fwd(h=ODD) == SHAPE and fwd(gp=ODD) == SHAPE
    assert fwd(T=0) == 0 and fwd(T=0, g=None, h=None) == 0

    need = lib.turnopd_block_norm_bwd_workspace_bytes(4, 64)
    assert need > 0 and lib.turnopd_block_norm_bwd_workspace_bytes(4, 0) == 0

    def bwd(resid=FAKE, rdt=1, ldr=64, rx=None, y=FAKE, ydt=1, ldy=64, yx=None, gp=FAKE, bp=None, gate=None, ldg=0, g=FAKE,
            T=4, d=64, kind=1, stats=FAKE, grdt=1, gydt=1, dh=FAKE, lddh=64, dro=FAKE, lddro=64, dr=ctypes.c_void_p(0x20000),
            lddr=64, dy=FAKE, lddy=64, dgate=None, lddg=64, dgp=FAKE, dbp=None, dg=FAKE, db=None, ws=FAKE, wsb=need, alpha=1.0):
        return lib.turnopd_block_norm_bwd(resid, rdt, ldr, rx, y, ydt, ldy, yx, gp, bp, gate, ldg, g, 1, None, T, d, kind,
                                          alpha, 1.0, stats, grdt, gydt, dh, lddh, dro, lddro, dr, lddr, dy, lddy, dgate, lddg,
                                          dgp, dbp, dg, db, ws, wsb, None)

    assert bwd(resid=None) == NULL and bwd(y=None) == NULL and bwd(stats=None) == NULL and bwd(dh=None) == NULL
    assert bwd(rdt=2) == NULL and bwd(ydt=3) == NULL  # codes need their exponents
    assert bwd(g=None, dg=None, dh=None, dro=None) == NULL
    assert bwd(dr=None, dy=None, dgp=None, dg=None) == NULL
    assert bwd(rdt=4) == UNSUPPORTED and bwd(grdt=2) == UNSUPPORTED and bwd(gydt=3) == UNSUPPORTED and bwd(kind=-1) == UNSUPPORTED
    assert bwd(dgate=FAKE) == UNSUPPORTED and bwd(gp=None) == UNSUPPORTED and bwd(g=None, dh=None) == UNSUPPORTED
    assert bwd(g=None, dg=None) == UNSUPPORTED    # dh without the norm it comes through
    assert bwd(dr=FAKE, lddr=72) == UNSUPPORTED   # in place needs one stride
    assert bwd(lddh=63) == SHAPE and bwd(lddro=63) == SHAPE and bwd(lddr=63) == SHAPE and bwd(lddy=63) == SHAPE
    assert bwd(gate=FAKE, ldg=64, dgate=FAKE, lddg=63) == SHAPE and bwd(stats=ctypes.c_void_p(0x10008)) == SHAPE
    assert bwd(dg=ODD) == SHAPE and bwd(dy=ODD) == SHAPE and bwd(alpha=INF) == SHAPE
    assert bwd(rdt=2, rx=FAKE, ldr=63) == SHAPE
    assert bwd(ws=None) == WORKSPACE and bwd(wsb=need - 1) == WORKSPACE and bwd(ws=ctypes.c_void_p(0x10010)) == WORKSPACE
    assert bwd(T=0, dgp=None, dg=None) == 0


def test_act8_host_validation(lib):
    def store(x=FAKE, dt=1, ldx=64, T=4, d=64, q=FAKE, code=2, ldc=64, exps=FAKE, status=FAKE):
        return lib.turnopd_act8_store(x, dt, ldx, None, T, d, q, code, ldc, exps, status, None)

    assert store(x=None) == NULL and store(q=None) == NULL and store(exps=None) == NULL and store(status=None) == NULL
    assert store(dt=2) == UNSUPPORTED and store(code=1) == UNSUPPORTED and store(code=4) == UNSUPPORTED
    assert store(ldx=63) == SHAPE and store(ldc=63) == SHAPE and store(d=0) == SHAPE and store(x=ODD) == SHAPE
    assert store(T=0) == 0

    def load(q=FAKE, code=3, ldc=64, exps=FAKE, T=4, d=64, out=FAKE, dt=0, ldo=64):
        return lib.turnopd_act8_load(q, code, ldc, exps, T, d, out, dt, ldo, None)

    assert load(q=None) == NULL and load(exps=None) == NULL and load(out=None) == NULL
    assert load(dt=3) == UNSUPPORTED and load(code=0) == UNSUPPORTED
    assert load(ldo=63) == SHAPE and load(ldc=63) == SHAPE and load(out=ODD) == SHAPE and load(T=-1) == SHAPE
    assert load(T=0) == 0


def test_binding_refuses_what_does_not_fit():
    import torch

    import paper_2607_05804_gb300 as P

    x, v, ids = torch.zeros(2, 8), torch.zeros(8), torch.zeros(2, dtype=torch.int32)
    with pytest.raises(ValueError):
        P.turnopd_embedding_fwd(x, ids, None, 1.0, x, None)
    with pytest.raises(ValueError):
        P.turnopd_embedding_bwd(x, ids, None, 1.0, x, 0, None, None)
    with pytest.raises(ValueError):
        P.turnopd_block_norm_fwd(x, x, v, None, None, v, None, None, 1, 1e-6, 1.0, 1.0, x, x, None, None)
    with pytest.raises(ValueError):
        P.turnopd_block_norm_bwd(x, x, v, None, None, v, None, 1, 1.0, 1.0, x, None, None, x, x, None, None, None, None, None,
                                 None)
    with pytest.raises(ValueError):
        P.turnopd_act8_store(x, None, x.to(torch.int8), x.to(torch.uint8), None)
    with pytest.raises(ValueError):
        P._param_dtype(v, v.half())
    with pytest.raises(ValueError):
        P._param_dtype(v.half())
    with pytest.raises(ValueError):
        P._act8_code(x, "codes")


def test_workspace_of_a_larger_batch_will_do(lib):
    """No batch needs more than a larger one, wherever the lengths of the tiles double."""
    for d in (1, 256, 1001, 4096, 8200, 3_000_000):
        for vocab in (100, 151_936):
            sizes = [lib.turnopd_embedding_bwd_workspace_bytes(T, d, vocab)
                     for T in sorted({k * n + j for n in (1, 2, 4, 8, 16, 32, 64) for k in (1, 97, 511, 1022, 4095, 8191, 8192, 65_536)
                                      for j in (0, 1, 15, 16)})]
            assert sizes == sorted(sizes) and sizes[0] > 0
    # partial sums of two rows of 4,096 columns for each of 1,022 tiles at most, beside the list of tokens
    assert lib.turnopd_embedding_bwd_workspace_bytes(32_768, 4096, 100) <= 1022 * 2 * 4096 * 4 + 32_768 * 16 + 1024
