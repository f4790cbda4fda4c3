"""The recognition operators' C entry points without a GPU: every refusal comes
before the first HIP call, with the documented status."""
import ctypes

import pytest

import paper_1410_4984_amd as gpps
from paper_1410_4984_amd import operators

OK, NULL, SHAPE, HYPER, DTYPE, WS, ALIGN, HIP, PATH = range(9)
FAKE = 0x7F0000000000        # never dereferenced
BIG = 1 << 40


def norm(dt=0, N=4, D=8, x=FAKE, ldx=8, w=FAKE, b=FAKE, eps=1e-5, y=FAKE, ldy=8, mean=FAKE, rstd=FAKE):
    return operators._lib().gpps_layer_norm(dt, N, D, x, ldx, w, b, eps, y, ldy, mean, rstd, None)


def norm_grads(dt=0, N=4, D=8, x=FAKE, ldx=8, w=FAKE, mean=FAKE, rstd=FAKE, dy=FAKE, lddy=8, dx=FAKE, lddx=8,
               dw=FAKE, db=FAKE, flags=0, ws=FAKE, n=BIG):
    return operators._lib().gpps_layer_norm_grads(dt, N, D, x, ldx, w, mean, rstd, dy, lddy, dx, lddx, dw, db, flags,
                                                  ws, n, None)


def rec(dt=0, N=4, B=2, D=8, x=FAKE, ldx=8, g=FAKE, ldg=8, off=FAKE, h0=FAKE, h=FAKE, ldh=8, last=FAKE, flags=0,
        ws=FAKE, n=BIG):
    return operators._lib().gpps_recurrence(dt, N, B, D, x, ldx, g, ldg, off, h0, h, ldh, last, flags, ws, n, None)


def rec_grads(dt=0, N=4, B=2, D=8, x=FAKE, ldx=8, g=FAKE, ldg=8, h=FAKE, ldh=8, dh=FAKE, lddh=8, off=FAKE, h0=FAKE,
              dlast=FAKE, dx=FAKE, lddx=8, dg=FAKE, lddg=8, dh0=FAKE, flags=0, ws=FAKE, n=BIG):
    return operators._lib().gpps_recurrence_grads(dt, N, B, D, x, ldx, g, ldg, h, ldh, dh, lddh, off, h0, dlast, dx,
                                                  lddx, dg, lddg, dh0, flags, ws, n, None)


@pytest.mark.parametrize("fn", [norm, norm_grads, rec, rec_grads])
def test_shapes_types_and_addresses(fn):
    assert fn(dt=3) == DTYPE and fn(dt=-1) == DTYPE
    assert fn(N=-1) == SHAPE and fn(D=0) == SHAPE and fn(D=16385) == SHAPE
    assert fn(N=1 << 39) == SHAPE                            # N D past 2^40
    assert fn(ldx=7) == SHAPE
    assert fn(x=None) == NULL
    assert fn(x=FAKE + 2) == ALIGN and fn(dt=2, x=FAKE + 1) == ALIGN and fn(dt=1, x=FAKE + 4) == ALIGN


def test_layer_norm():
    assert norm(ldy=7) == SHAPE and norm(y=None) == NULL
    for eps in (float("nan"), float("inf"), -1e-9):
        assert norm(eps=eps) == HYPER
    # weights and statistics are in 32 bits beside bfloat16 rows
    for k in ("w", "b", "mean", "rstd"):
        assert norm(dt=2, **{k: FAKE + 2}) == ALIGN
    assert norm(N=0, x=None, y=None) == OK                   # nothing to do, nothing launched
    for k in ("mean", "rstd", "dy", "dx", "ws"):
        assert norm_grads(**{k: None}) == NULL, k
    assert norm_grads(lddy=7) == SHAPE and norm_grads(lddx=7) == SHAPE
    assert norm_grads(flags=2) == PATH and norm_grads(flags=16) == PATH
    need = operators._lib().gpps_layer_norm_workspace_bytes(0, 4, 8)
    assert need > 0 and norm_grads(n=need - 1) == WS and norm_grads(ws=FAKE + 64) == ALIGN
    assert operators._lib().gpps_layer_norm_workspace_bytes(0, 4, 0) == 0
    assert operators._lib().gpps_layer_norm_workspace_bytes(5, 4, 8) == 0


def test_recurrence():
    for fn in (rec, rec_grads):
        assert fn(B=0) == SHAPE and fn(B=1 << 31) == SHAPE
        assert fn(off=None) == SHAPE                         # two sequences need offsets
        assert fn(N=(1 << 36) + 1, D=1) == SHAPE             # past the tiles' counter
        assert fn(off=FAKE + 4) == ALIGN
        assert fn(g=None) == NULL and fn(h=None) == NULL and fn(ws=None) == NULL
        assert fn(ldg=7) == SHAPE and fn(ldh=7) == SHAPE
        assert fn(flags=1) == PATH and fn(flags=16) == PATH
        assert fn(dt=2, h0=FAKE + 2) == ALIGN
        need = operators._lib().gpps_recurrence_workspace_bytes(0, 4, 2, 8)
        assert need > 0 and fn(n=need - 1) == WS and fn(ws=FAKE + 8) == ALIGN
    assert rec_grads(dx=None) == NULL and rec_grads(dg=None) == NULL
    assert rec_grads(lddx=7) == SHAPE and rec_grads(lddg=7) == SHAPE and rec_grads(lddh=7) == SHAPE
    assert rec_grads(dh0=FAKE + 2) == ALIGN
    assert operators._lib().gpps_recurrence_workspace_bytes(0, 4, 0, 8) == 0


def adam(dt=0, gdt=0, bits=32, sizes=(3, 4), p=FAKE, g=FAKE, m=FAKE, v=FAKE, ms=None, vs=None, step=1, lr=1e-3,
         b1=0.9, b2=0.99, eps=1e-8, wd=0.0, flags=0, count=None):
    k = len(sizes)
    ptrs = [(ctypes.c_void_p * k)(*[q] * k) if q is None or q > 1 else None for q in (p, g, m, v, ms, vs)]
    return operators._lib().gpps_adamw(dt, gdt, bits, k if count is None else count, (ctypes.c_int64 * k)(*sizes),
                                       *ptrs, step, lr, b1, b2, eps, wd, flags, None)


def test_adamw():
    assert adam(dt=3) == DTYPE and adam(gdt=1) == DTYPE and adam(dt=1, gdt=0, bits=64) == DTYPE
    assert adam(bits=16) == DTYPE and adam(bits=64) == DTYPE and adam(dt=1, gdt=1, bits=8) == DTYPE
    assert adam(dt=1, gdt=1, bits=32) == DTYPE
    assert adam(count=-1) == SHAPE and adam(step=0) == SHAPE and adam(sizes=(3, -1)) == SHAPE
    for k in "pgmv":
        assert adam(**{k: None}) == NULL and adam(**{k: 0}) == NULL, k
    assert adam(bits=8, ms=FAKE) == NULL and adam(bits=8, vs=FAKE) == NULL
    assert adam(p=FAKE + 2) == ALIGN and adam(m=FAKE + 2) == ALIGN and adam(bits=8, ms=FAKE + 2, vs=FAKE) == ALIGN
    nan, inf = float("nan"), float("inf")
    for bad in ({"lr": nan}, {"lr": inf}, {"lr": -1.0}, {"b1": 1.0}, {"b1": -0.1}, {"b2": nan}, {"eps": -1.0},
                {"eps": inf}, {"wd": -1.0}, {"wd": nan}):
        assert adam(**bad) == HYPER, bad
    assert adam(flags=1) == PATH
    assert adam(sizes=(0, 0), p=None, g=None, m=None, v=None) == OK     # nothing to do
    assert adam(sizes=(), count=0) == OK
    L = operators._lib()
    assert L.gpps_adamw_values(2, 4, FAKE, FAKE, FAKE, None) == SHAPE
    assert L.gpps_adamw_values(0, -1, FAKE, FAKE, FAKE, None) == SHAPE
    assert L.gpps_adamw_values(0, 4, None, FAKE, FAKE, None) == NULL
    assert L.gpps_adamw_values(0, 4, FAKE, FAKE + 2, FAKE, None) == ALIGN
    assert L.gpps_adamw_values(0, 0, None, None, None, None) == OK


def test_the_other_calls_refuse_bfloat16():
    assert gpps.lib().gpps_workspace_bytes(2, 10, 4, 2) == 0
    l = (ctypes.c_double * 2)(1.0, 1.0)
    assert gpps.lib().gpps_psi_stats(2, 10, 4, 2, FAKE, FAKE, FAKE, 1.0, l, FAKE, FAKE, FAKE, 0, FAKE, BIG, None) == DTYPE


def test_binding_refuses_cpu_tensors():
    torch = pytest.importorskip("torch")
    x = torch.zeros(4, 3)
    for call in (lambda: gpps.layer_norm(x), lambda: gpps.recurrence(x, x),
                 lambda: gpps.adamw_step([x], [x], [x.clone()], [x.clone()], 1, 1e-3)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(ValueError):
        gpps.AdamW([x], bits=16)
