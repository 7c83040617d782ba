"""Host-side argument checks of the token log probabilities and the norm (they return before any CUDA call)."""
import ctypes

import pytest

FAKE = ctypes.c_void_p(0x10000)  # never dereferenced: every call below fails validation first
ODD = ctypes.c_void_p(0x10001)


@pytest.fixture(scope="module")
def lib():
    from paper_2607_05804_gb300 import build as B

    B.build()
    import paper_2607_05804_gb300 as P

    return P.load()


def test_logprobs_host_validation(lib):
    need = lib.turnopd_token_logprobs_workspace_bytes(64)
    assert need >= 64 * 16 and lib.turnopd_token_logprobs_workspace_bytes(-1) == 0

    def call(z=FAKE, dt=1, ld=1024, vocab=1024, rows=64, rot=None, y=FAKE, mask=FAKE, T=64, n_top=5, lp=FAKE, ent=FAKE,
             stats=FAKE, tid=FAKE, tlp=FAKE, ws=FAKE, wsb=need, status=FAKE):
        return lib.turnopd_token_logprobs(z, dt, ld, vocab, rows, rot, y, mask, T, n_top, lp, ent, stats, tid, tlp, ws,
                                          wsb, status, None)

    assert call(status=None) == 1 and call(z=None) == 1
    assert call(y=None) == 1                       # a log probability needs its token
    assert call(tid=None) == 1 and call(tlp=None) == 1
    assert call(lp=None, ent=None, stats=None, n_top=0) == 1
    assert call(dt=2) == 6
    assert call(ld=1023) == 2 and call(vocab=0) == 2 and call(rows=63) == 2 and call(T=-1) == 2
    assert call(n_top=33) == 2 and call(n_top=-1) == 2 and call(n_top=5, vocab=4) == 2
    assert call(z=ODD) == 2 and call(lp=ODD) == 2 and call(tid=ODD) == 2
    assert call(ws=None) == 10 and call(wsb=need - 1) == 10 and call(ws=ctypes.c_void_p(0x10010)) == 10
    # nothing to do: no launch, with and without a mask
    assert call(T=0, rows=0, z=None) == 0
    assert call(T=0, rows=0, z=None, mask=None, ws=None, wsb=0) == 0


def test_logprobs_bwd_host_validation(lib):
    need = lib.turnopd_token_logprobs_workspace_bytes(64)

    def call(z=FAKE, dt=1, ld=1024, vocab=1024, rows=64, y=FAKE, mask=FAKE, T=64, stats=FAKE, lp=FAKE, ent=FAKE, gl=FAKE,
             gh=FAKE, g=ctypes.c_void_p(0x20000), gdt=1, flags=0, ws=FAKE, wsb=need, status=FAKE):
        return lib.turnopd_token_logprobs_bwd(z, dt, ld, vocab, rows, None, y, mask, T, stats, lp, ent, gl, gh, g, gdt,
                                              flags, ws, wsb, status, None)

    assert call(status=None) == 1 and call(g=None) == 1 and call(stats=None) == 1
    assert call(gl=None, gh=None) == 1
    assert call(y=None) == 1 and call(lp=None) == 1 and call(ent=None) == 1
    assert call(dt=7) == 6 and call(gdt=7) == 6 and call(flags=0x100) == 6
    assert call(g=FAKE, gdt=0) == 6                # in place needs one type
    assert call(ld=1000) == 2 and call(g=ODD) == 2 and call(gl=ODD) == 2
    assert call(ws=None) == 10 and call(wsb=need - 1) == 10
    assert call(T=0, rows=0) == 0


def test_norm_host_validation(lib):
    def fwd(x=FAKE, xdt=1, ldx=64, gamma=FAKE, beta=None, pdt=1, T=4, d=64, kind=0, eps=1e-6, y=FAKE, ydt=1, ldy=64,
            mean=None, rstd=None, status=FAKE):
        return lib.turnopd_norm_fwd(x, xdt, ldx, gamma, beta, pdt, None, T, d, kind, eps, y, ydt, ldy, mean, rstd, status,
                                    None)

    assert fwd(x=None) == 1 and fwd(y=None) == 1 and fwd(gamma=None) == 1 and fwd(status=None) == 1
    assert fwd(xdt=3) == 6 and fwd(ydt=3) == 6 and fwd(pdt=3) == 6 and fwd(kind=2) == 6
    assert fwd(d=0) == 2 and fwd(ldx=63) == 2 and fwd(ldy=63) == 2 and fwd(T=-1) == 2
    assert fwd(eps=-1e-6) == 2 and fwd(eps=float("nan")) == 2 and fwd(eps=float("inf")) == 2
    assert fwd(x=ODD) == 2 and fwd(y=ODD) == 2 and fwd(gamma=ODD) == 2 and fwd(mean=ODD) == 2
    assert fwd(T=0) == 0

    need = lib.turnopd_norm_bwd_workspace_bytes(4, 64)
    assert need > 0 and lib.turnopd_norm_bwd_workspace_bytes(4, 0) == 0

    def bwd(x=FAKE, ldx=64, gamma=FAKE, T=4, d=64, kind=0, mean=FAKE, rstd=FAKE, dy=FAKE, dydt=0, lddy=64, dx=FAKE, dxdt=1,
            lddx=64, dg=FAKE, db=FAKE, ws=FAKE, wsb=need):
        return lib.turnopd_norm_bwd(x, 1, ldx, gamma, 1, None, T, d, kind, mean, rstd, dy, dydt, lddy, dx, dxdt, lddx, dg,
                                    db, ws, wsb, None)

    assert bwd(x=None) == 1 and bwd(dy=None) == 1 and bwd(rstd=None) == 1 and bwd(mean=None) == 1 and bwd(gamma=None) == 1
    assert bwd(dx=None, dg=None, db=None) == 1
    assert bwd(dydt=5) == 6 and bwd(dxdt=5) == 6 and bwd(kind=-1) == 6
    assert bwd(lddy=63) == 2 and bwd(lddx=63) == 2 and bwd(dg=ODD) == 2 and bwd(mean=ODD) == 2
    assert bwd(ws=None) == 10 and bwd(wsb=need - 1) == 10 and bwd(ws=ctypes.c_void_p(0x10010)) == 10
    assert bwd(T=0, dg=None, db=None) == 0


def test_binding_refuses_host_tensors():
    import torch

    import paper_2607_05804_gb300 as P

    z = torch.zeros(2, 8)
    with pytest.raises(ValueError):
        P.turnopd_token_logprobs(z, 8, None, None, None, 0, None, z[0], None, None, None, None, None)
    with pytest.raises(ValueError):
        P.turnopd_norm_fwd(z, z[0], None, None, 0, 1e-6, z, None, None, None)
