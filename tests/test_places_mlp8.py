"""Where results of the MLP operators may lie: apart from the operands, or in place of one that the same lane reads element for
element. Everything else is refused on the host, since blocks write while others still read (no call here reaches a device)."""
import ctypes
import itertools

import pytest

from paper_2608_24070_amd import slim

A = 1 << 20          # addresses 16 MiB apart (never dereferenced): every operand here is smaller
at = lambda i: (i + 1) * (A << 4)
BF16, F32, Q8 = slim.SLIM_BF16, slim.SLIM_F32, slim.SLIM_Q8_E4M3
INV = slim.SLIM_EINVAL
M, N, K = 70, 192, 256


class Rows(ctypes.Structure):
    _fields_ = [("at", ctypes.c_void_p), ("rows", ctypes.c_int64), ("bytes", ctypes.c_int64), ("step", ctypes.c_int64)]


def test_rows_that_meet():
    f = slim.lib()._Z14slim_rows_meetRK8SlimRowsS1_
    f.restype = ctypes.c_bool
    meet = lambda a, b: bool(f(ctypes.byref(Rows(*a)), ctypes.byref(Rows(*b))))
    cells = lambda r: {r[0] + i * r[3] + j for i in range(r[1]) for j in range(r[2])}
    shapes = [(rows, width, step) for rows in (1, 2, 3) for width in (1, 2, 4) for step in (4, 5, 9)]
    for (ra, wa, sa), (rb, wb, sb) in itertools.product(shapes, shapes):
        for off in range(-24, 25):
            a, b = (100, ra, wa, sa), (100 + off, rb, wb, sb)
            assert meet(a, b) == bool(cells(a) & cells(b)), (a, b)
    # nothing there; steps and counts whose product passes 64 bits
    assert not meet((None, 5, 8, 8), (None, 5, 8, 8)) and not meet((4096, 0, 8, 8), (4096, 5, 8, 8))
    assert meet((4096, 1 << 40, 8, 1 << 40), (4096 + (5 << 40), 3, 8, 8)) and not meet((4096, 1 << 40, 8, 1 << 40), (4104 + (5 << 40), 3, 8, 8))


def forward(kw):
    a = dict(dict(X=at(0), xdt=BF16, xe=at(1), ldx=K, bias=at(2), mul=at(3), ldm=N, res=at(4), ldr=N, q8=0, Y=at(5), ldy=N, ye=at(6), pre=at(7),
                  ldp=N, pe=at(8), M=M), **kw)
    need = slim.slim_linear8_act_workspace(a["xdt"], a["M"], N, K, BF16, a["q8"])
    return slim.slim_linear8_act(a["X"], a["xdt"], a["xe"], a["M"], N, K, a["ldx"], at(9), at(10), slim.SLIM_ACT_GELU, a["bias"], F32, a["mul"],
                                 a["ldm"], a["res"], a["ldr"], BF16, a["q8"], a["Y"], a["ldy"], a["ye"], a["pre"], a["ldp"], a["pe"], at(11), need,
                                 None)


@pytest.mark.parametrize("kw", [
    # 8-bit results over 16-bit operands
    dict(q8=1, Y=at(3)), dict(q8=1, Y=at(4)), dict(q8=1, pre=at(3)), dict(q8=1, pre=at(4)), dict(q8=1, Y=at(3) + 16 * N), dict(q8=1, ye=at(4) + 2 * N),
    # the rows' own place at another stride, a row or a column further, or so that only the last rows meet
    dict(Y=at(3), ldy=N + 8), dict(Y=at(4), ldr=2 * N), dict(pre=at(3), ldp=N + 1), dict(Y=at(3) + 2 * N), dict(Y=at(4) + 2),
    dict(Y=at(3) + 2 * N * (M - 1)), dict(Y=at(4) - 2 * N * (M - 1)), dict(mul=at(3), ldm=2 * N, Y=at(3) + N, ldy=2 * N),
    # X and its exponents, in whole or in part; the bias
    dict(Y=at(0)), dict(pre=at(0)), dict(Y=at(0) + 2 * K * (M - 1)), dict(xdt=Q8, Y=at(0) + 128), dict(xdt=Q8, Y=at(1)), dict(xdt=Q8, q8=1, ye=at(1)),
    dict(xdt=Q8, q8=1, pe=at(1) + 16), dict(M=2, ldx=K, Y=at(0) + 2 * K), dict(Y=at(2)), dict(pre=at(2) - 2 * N * (M - 1)),
    # each other
    dict(pre=at(5)), dict(pre=at(5) + 2), dict(pre=at(5) + 2 * N, ldp=3 * N), dict(q8=1, pre=at(5)), dict(q8=1, pe=at(6)), dict(q8=1, ye=at(5) + 256)])
def test_forward(kw):
    assert forward(kw) == INV


# places, of [M, K]: U, mul in 16 bits (K columns, ld) or in 8 bits; exponents are Q8's only
BWD = [
    # 16-bit results over 8-bit operands or their exponents
    dict(udt=Q8, dU=at(2)), dict(udt=Q8, dmul=at(4)), dict(udt=Q8, dU=at(4)), dict(udt=Q8, dmul=at(2) + 16 * K), dict(udt=Q8, dU=at(3)),
    dict(udt=Q8, dmul=at(5)), dict(udt=Q8, db=at(2)),
    # an operand's own place at another stride, a row or a column further, or so that only the last rows meet
    dict(dU=at(2), ldo=K + 8), dict(dmul=at(4), ldm=2 * K), dict(dU=at(2) + 2 * K), dict(dU=at(4) + 2), dict(dmul=at(2) + 2 * K * (M - 1)),
    dict(dU=at(4) - 2 * K * (M - 1)), dict(db=at(2) + 2 * K), dict(db=at(4)),
    # each other
    dict(dmul=at(6)), dict(dmul=at(6) + 2), dict(dmul=at(6) + 2 * K, ldd=3 * K), dict(db=at(6)), dict(db=at(7) + 2 * K * (M - 1)),
    dict(dU=at(2), dmul=at(2)), dict(M=1, db=at(6)), dict(M=1, dmul=at(6) + K)]


@pytest.mark.parametrize("kw", BWD + [
    # dY where blocks read it as it is
    dict(xdt=Q8, dU=at(0)), dict(xdt=Q8, dmul=at(0)), dict(xdt=Q8, dU=at(0) + 128), dict(xdt=Q8, dU=at(1)), dict(xdt=Q8, db=at(0))])
def test_bwd_dx8_act(kw):
    a = dict(dict(X=at(0), xdt=BF16, xe=at(1), U=at(2), ue=at(3), ldu=K, mul=at(4), me=at(5), ldm=K, udt=BF16, dU=at(6), ldo=K, dmul=at(7), ldd=K,
                  db=at(8), M=M), **kw)
    need = slim.slim_bwd_dx8_act_workspace(a["xdt"], a["M"], N, K, BF16, 1)
    assert slim.slim_bwd_dx8_act(a["X"], a["xdt"], a["xe"], a["M"], N, K, N, at(9), at(10), slim.SLIM_ACT_GELU, a["U"], a["udt"], a["ue"], a["ldu"],
                                 a["mul"], a["me"], a["ldm"], BF16, a["dU"], a["ldo"], a["dmul"], a["ldd"], a["db"], at(11), need, None) == INV


@pytest.mark.parametrize("kw", BWD + [dict(dU=at(0), ldx=K + 1), dict(dmul=at(0) + 2 * K), dict(dU=at(0), dmul=at(0)), dict(db=at(0))])
def test_act_bwd(kw):
    a = dict(dict(X=at(0), ldx=K, U=at(2), ue=at(3), ldu=K, mul=at(4), me=at(5), ldm=K, udt=BF16, dU=at(6), ldo=K, dmul=at(7), ldd=K, db=at(8), M=M),
             **kw)
    need = slim.slim_act_bwd_workspace(a["M"], K, 1)
    assert slim.slim_act_bwd(a["X"], BF16, a["ldx"], a["M"], K, slim.SLIM_ACT_GELU, a["U"], a["udt"], a["ue"], a["ldu"], a["mul"], a["me"], a["ldm"],
                             a["dU"], a["ldo"], a["dmul"], a["ldd"], a["db"], at(11), need, None) == INV


@pytest.mark.parametrize("kw", [
    # the residual's rows at another stride, or a part of them; what other blocks look up
    dict(Y=at(2), ldy=K + 8), dict(Y=at(2), ldr=2 * K), dict(Y=at(2) + 2 * K), dict(Y=at(2) + 2), dict(Y=at(2) - 2 * K * 6), dict(Y=at(3)),
    dict(Y=at(4)), dict(Y=at(3) - 2 * K * 6), dict(M=1, Y=at(3)), dict(M=1, Y=at(2) + K)])
def test_moe8(kw):
    a = dict(dict(M=7, X=at(0), res=at(2), ldr=K, Y=at(5), ldy=K), **kw)
    need = slim.slim_moe8_workspace(a["M"], K, 300, 40, 4)
    assert slim.slim_moe8(a["X"], BF16, None, a["M"], K, K, 300, 40, at(6), at(7), at(8), at(9), at(10), at(11), slim.SLIM_ACT_SILU, at(3), at(4), 4,
                          a["res"], a["ldr"], a["Y"], BF16, a["ldy"], at(12), need, None) == INV
