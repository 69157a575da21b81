"""The 8-bit path's entry points refuse bad arguments on the host (no call here reaches a device), and the binding refuses
tensors that do not fit before it makes a pointer of them."""
import re

import pytest
import torch

from paper_2608_24070_amd import slim

A = 1 << 20          # a fake, 16-byte aligned, non-null "device" address (never dereferenced)
ODD = A + 1          # no element of any type starts here
MIS = A + 8          # an element, but not 16-byte aligned
F16, BF16, F32, Q8 = slim.SLIM_F16, slim.SLIM_BF16, slim.SLIM_F32, slim.SLIM_Q8_E4M3
INV, SHAPE, DTYPE, ALIGN, WS, UNSUP = (slim.SLIM_EINVAL, slim.SLIM_ESHAPE, slim.SLIM_EDTYPE, slim.SLIM_EALIGN,
                                       slim.SLIM_EWORKSPACE, slim.SLIM_EUNSUPPORTED)
WIDE = (1 << 22) + 1


def test_type_code_matches_header():
    assert int(re.search(r"SLIM_Q8_E4M3 = (\d+)", open(slim.HEADER).read()).group(1)) == Q8
    assert {"slim_quant8", "slim_dequant8", "slim_pack8", "slim_linear8_workspace", "slim_linear8", "slim_grad_w8",
            "slim_norm", "slim_norm_bwd_workspace", "slim_norm_bwd"} <= set(slim.header_symbols())


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(codes=None), INV), (dict(exps=None), INV), (dict(dtype=Q8), DTYPE), (dict(dtype=7), DTYPE),
    (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(ldx=99), SHAPE), (dict(K=WIDE, ldx=WIDE), SHAPE), (dict(X=ODD), ALIGN),
    (dict(dtype=F32, X=A + 2), ALIGN), (dict(codes=MIS), ALIGN), (dict(exps=MIS), ALIGN),
    (dict(M=1 << 32), UNSUP), (dict(M=0, X=None), slim.SLIM_OK)])
def test_quant8(kw, status):
    a = dict(dict(X=A, dtype=F16, M=3, K=100, ldx=100, codes=A, exps=A), **kw)
    assert slim.slim_quant8(a["X"], a["dtype"], a["M"], a["K"], a["ldx"], a["codes"], a["exps"], None) == status
    # the way back has the same rules
    assert slim.slim_dequant8(a["codes"], a["exps"], a["M"], a["K"], a["X"], a["dtype"], a["ldx"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(W=None), INV), (dict(codes=None), INV), (dict(exps=None), INV), (dict(codesT=A), INV), (dict(expsT=A), INV),
    (dict(codes=None, exps=None), INV), (dict(dtype=Q8), DTYPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(ldw=99), SHAPE),
    (dict(N=WIDE), SHAPE), (dict(W=A + 2), ALIGN), (dict(codes=MIS), ALIGN), (dict(codesT=MIS, expsT=A), ALIGN)])
def test_pack8(kw, status):
    a = dict(dict(W=A, dtype=F32, N=10, K=100, ldw=100, codes=A, exps=A, codesT=None, expsT=None), **kw)
    assert slim.slim_pack8(a["W"], a["dtype"], a["N"], a["K"], a["ldw"], a["codes"], a["exps"], a["codesT"], a["expsT"],
                           None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(xexps=None, xdt=Q8), INV), (dict(codes=None), INV), (dict(exps=None), INV), (dict(Y=None), INV),
    (dict(xdt=5), DTYPE), (dict(ydt=F32), DTYPE), (dict(ydt=Q8), DTYPE), (dict(M=-1), SHAPE), (dict(N=0), SHAPE),
    (dict(K=0), SHAPE), (dict(ldx=255), SHAPE), (dict(ldy=19), SHAPE), (dict(N=WIDE, ldy=WIDE), SHAPE), (dict(X=ODD), ALIGN),
    (dict(X=MIS, xdt=Q8), ALIGN), (dict(codes=MIS), ALIGN), (dict(Y=ODD), ALIGN), (dict(ws=None), WS), (dict(short=1), WS),
    (dict(ws=MIS), ALIGN), (dict(M=1 << 32), UNSUP), (dict(M=0, X=None), slim.SLIM_OK)])
def test_linear8(kw, status):
    a = dict(dict(X=A, xdt=BF16, xexps=A, M=70, N=20, K=256, ldx=256, codes=A, exps=A, Y=A, ydt=BF16, ldy=20, ws=A, short=0), **kw)
    try:
        need = slim.slim_linear8_workspace(a["xdt"], a["M"], a["N"], a["K"])
    except slim.SlimError as e:
        assert e.status == status
        need = 1 << 40
    assert slim.slim_linear8(a["X"], a["xdt"], a["xexps"], a["M"], a["N"], a["K"], a["ldx"], a["codes"], a["exps"], a["Y"],
                             a["ydt"], a["ldy"], a["ws"], need - a["short"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dY=None), INV), (dict(xc=None), INV), (dict(xe=None), INV), (dict(gW=None), INV), (dict(dt=F32), DTYPE), (dict(dt=Q8), DTYPE),
    (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE), (dict(lddy=9), SHAPE), (dict(meta=A, K=40), SHAPE), (dict(N=WIDE, lddy=WIDE), SHAPE),
    (dict(dY=ODD), ALIGN), (dict(xc=MIS), ALIGN), (dict(xe=MIS), ALIGN), (dict(gW=MIS), ALIGN), (dict(meta=MIS, K=32), ALIGN), (dict(ws=None), WS), (dict(short=1), WS), (dict(ws=MIS), ALIGN), (dict(M=1 << 31), UNSUP)])
def test_grad_w8(kw, status):
    a = dict(dict(dY=A, dt=BF16, lddy=10, xc=A, xe=A, M=5000, N=10, K=36, meta=None, gW=A, ws=A, short=0), **kw)
    try:
        need = slim.slim_grad_w8_workspace(a["M"], a["N"], a["K"], int(a["meta"] is not None), 0)
    except slim.SlimError as e:
        assert e.status == status
        need = 1 << 40
    assert slim.slim_grad_w8(a["dY"], a["dt"], a["lddy"], a["xc"], a["xe"], a["M"], a["N"], a["K"], a["meta"], a["gW"], a["ws"],
                             need - a["short"], None) == status


def test_grad_w8_workspace_is_for_odd_rows_and_short_layers():
    assert slim.slim_grad_w8_workspace(8192, 28672, 8192, 1, 1) == 0
    assert slim.slim_grad_w8_workspace(1000, 8193, 8192, 0, 0) == -(-1000 * 8208 * 2 // 256) * 256
    assert slim.slim_grad_w8_workspace(8192, 128, 128, 0, 1) > 0 and slim.slim_grad_w8_workspace(0, 128, 128, 0, 0) == 0


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(Y=None), INV), (dict(rstd=None), INV), (dict(ydt=Q8, ye=None), INV), (dict(eps=-1.0), INV),
    (dict(eps=float("nan")), INV), (dict(rms=1), INV), (dict(dt=Q8), DTYPE), (dict(pdt=Q8), DTYPE), (dict(ydt=F32), DTYPE), (dict(M=-1), SHAPE),
    (dict(K=0), SHAPE), (dict(ldx=9), SHAPE), (dict(ldy=9), SHAPE), (dict(K=WIDE, ldx=WIDE, ldy=WIDE), SHAPE), (dict(X=ODD), ALIGN),
    (dict(Y=MIS, ydt=Q8), ALIGN), (dict(gamma=A + 2), ALIGN), (dict(mean=A + 2), ALIGN), (dict(rstd=A + 2), ALIGN), (dict(M=0, X=None), slim.SLIM_OK)])
def test_norm(kw, status):
    a = dict(dict(X=A, dt=F16, M=3, K=10, ldx=10, gamma=A, beta=A, pdt=F32, rms=0, eps=1e-5, Y=A, ydt=F16, ldy=10, ye=A, mean=A, rstd=A), **kw)
    assert slim.slim_norm(a["X"], a["dt"], a["M"], a["K"], a["ldx"], a["gamma"], a["beta"], a["pdt"], a["rms"], a["eps"], a["Y"],
                          a["ydt"], a["ldy"], a["ye"], a["mean"], a["rstd"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(dY=None), INV), (dict(X=None), INV), (dict(rstd=None), INV), (dict(dX=None), INV), (dict(xdt=Q8, xe=None), INV), (dict(dt=Q8), DTYPE),
    (dict(xdt=F32), DTYPE), (dict(pdt=9), DTYPE), (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(lddy=9), SHAPE), (dict(ldx=9), SHAPE),
    (dict(lddx=9), SHAPE), (dict(dY=ODD), ALIGN), (dict(X=MIS, xdt=Q8), ALIGN), (dict(dg=A + 2), ALIGN), (dict(ws=None), WS), (dict(short=1), WS),
    (dict(ws=MIS), ALIGN)])
def test_norm_bwd(kw, status):
    a = dict(dict(dY=A, dt=F16, lddy=10, X=A, xdt=F16, xe=A, ldx=10, M=30, K=10, gamma=A, pdt=F32, mean=A, rstd=A, dX=A, lddx=10, dg=A, db=A,
                  ws=A, short=0), **kw)
    try:
        need = slim.slim_norm_bwd_workspace(a["M"], a["K"])
    except slim.SlimError as e:
        assert e.status == status
        need = 1 << 40
    assert slim.slim_norm_bwd(a["dY"], a["dt"], a["lddy"], a["X"], a["xdt"], a["xe"], a["ldx"], a["M"], a["K"], a["gamma"], a["pdt"], a["mean"],
                              a["rstd"], a["dX"], a["lddx"], a["dg"], a["db"], a["ws"], need - a["short"], None) == status


def test_binding_refuses_host_tensors():
    x = torch.zeros(2, 256, dtype=torch.float16)
    for call in (lambda: slim.quant8(x), lambda: slim.pack8(x), lambda: slim.norm(x),
                 lambda: slim.norm_bwd(x, x, None, None, torch.zeros(2))):
        with pytest.raises(ValueError):
            call()


def test_sizes_past_one_launch():
    # eight threads a group of 128, and fewer than 2^32 threads a launch: refused before anything is read
    for m, k, status in ((1 << 29, 128, UNSUP), (1 << 22, 128 << 7, UNSUP), (1 << 29, 1, UNSUP)):
        assert slim.slim_quant8(A, F16, m, k, k, A, A, None) == status
        assert slim.slim_dequant8(A, A, m, k, A, F16, k, None) == status
    for xdt, m, n, k in ((BF16, 1 << 22, 16, 128 << 7), (Q8, 1 << 25, 16, 128 << 7)):
        with pytest.raises(slim.SlimError) as e:
            slim.slim_linear8_workspace(xdt, m, n, k)
        assert e.value.status == UNSUP
    # the pieces of a copy of dY are counted in 32 bits
    for m, n in (((1 << 31) - 1, 128), (1 << 20, 1 << 16)):
        with pytest.raises(slim.SlimError) as e:
            slim.slim_grad_w8_workspace(m, n, 128, 0, 0)
        assert e.value.status == UNSUP
    # a block of 1024 threads a row
    assert slim.slim_norm(A, F16, 1 << 22, 16385, 16385, None, None, F32, 0, 1e-5, A, F16, 16385, None, None, A, None) == UNSUP
    with pytest.raises(slim.SlimError) as e:
        slim.slim_norm_bwd_workspace(1 << 22, 16385)
    assert e.value.status == UNSUP
