"""The MLP operators' entry points refuse bad arguments on the host (no call here reaches a device), and the binding refuses tensors
that do not fit before it makes a pointer of them."""
import re

import pytest
import torch

from paper_2608_24070_amd import slim
from tests.test_binding8 import OnGpu

A = 1 << 20          # a fake, 16-byte aligned, non-null "device" address (never dereferenced)
ODD = A + 1          # no element of any type starts here
MIS = A + 8          # an element, but not 16-byte aligned
F16, BF16, F32, Q8 = slim.SLIM_F16, slim.SLIM_BF16, slim.SLIM_F32, slim.SLIM_Q8_E4M3
OK, INV, SHAPE, DTYPE, ALIGN, WS, UNSUP = (slim.SLIM_OK, slim.SLIM_EINVAL, slim.SLIM_ESHAPE, slim.SLIM_EDTYPE, slim.SLIM_EALIGN,
                                           slim.SLIM_EWORKSPACE, slim.SLIM_EUNSUPPORTED)
WIDE = (1 << 22) + 1


def test_codes_match_the_header():
    text = open(slim.HEADER).read()
    for name, code in slim.ACTS.items():
        assert int(re.search(rf"SLIM_ACT_{name.upper()} = (\d+)", text).group(1)) == code
    assert {"slim_linear8_act_workspace", "slim_linear8_act", "slim_bwd_dx8_act_workspace", "slim_bwd_dx8_act", "slim_act_bwd_workspace",
            "slim_act_bwd", "slim_route_workspace", "slim_route", "slim_moe8_workspace", "slim_moe8"} <= set(slim.header_symbols())


def needed(query, *args, status):
    """Workspace bytes; where the query refuses, it does with the call's status."""
    try:
        return query(*args)
    except slim.SlimError as e:
        assert e.status == status
        return 1 << 40


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(xexps=None, xdt=Q8), INV), (dict(codes=None), INV), (dict(exps=None), INV), (dict(Y=None), INV),
    (dict(act=5), INV), (dict(act=-1), INV), (dict(q8=1, yexps=None), INV), (dict(q8=1, preexps=None), INV), (dict(xdt=5), DTYPE),
    (dict(dt=F32), DTYPE), (dict(dt=Q8), DTYPE), (dict(bdt=Q8), DTYPE), (dict(M=-1), SHAPE), (dict(N=0), SHAPE), (dict(K=0), SHAPE),
    (dict(ldx=255), SHAPE), (dict(ldy=19), SHAPE), (dict(ldm=19), SHAPE), (dict(ldr=19), SHAPE), (dict(ldp=19), SHAPE),
    (dict(N=WIDE, ldy=WIDE), SHAPE), (dict(X=ODD), ALIGN), (dict(X=MIS, xdt=Q8), ALIGN), (dict(codes=MIS), ALIGN), (dict(Y=ODD), ALIGN),
    (dict(Y=MIS, q8=1), ALIGN), (dict(pre=MIS, q8=1), ALIGN), (dict(mul=ODD), ALIGN), (dict(res=ODD), ALIGN), (dict(bias=A + 2), ALIGN),
    (dict(ws=None), WS), (dict(short=1), WS), (dict(ws=MIS), ALIGN), (dict(M=1 << 32), UNSUP), (dict(M=0, X=None, Y=None), OK),
    (dict(Y=2 * A), INV), (dict(pre=2 * A), INV), (dict(pre=3 * A), INV)])
def test_linear8_act(kw, status):
    a = dict(dict(X=2 * A, xdt=BF16, xexps=A, M=70, N=20, K=256, ldx=256, codes=A, exps=A, act=2, bias=A, bdt=F32, mul=A, ldm=20, res=A, ldr=20,
                  dt=BF16, q8=0, Y=3 * A, ldy=20, yexps=A, pre=A, ldp=20, preexps=A, ws=A, short=0), **kw)
    need = needed(slim.slim_linear8_act_workspace, a["xdt"], a["M"], a["N"], a["K"], a["dt"], a["q8"], status=status)
    assert slim.slim_linear8_act(a["X"], a["xdt"], a["xexps"], a["M"], a["N"], a["K"], a["ldx"], a["codes"], a["exps"], a["act"], a["bias"],
                                 a["bdt"], a["mul"], a["ldm"], a["res"], a["ldr"], a["dt"], a["q8"], a["Y"], a["ldy"], a["yexps"], a["pre"],
                                 a["ldp"], a["preexps"], a["ws"], need - a["short"], None) == status


BWD = [(dict(U=None), INV), (dict(U=None, act=0), INV), (dict(dU=None), INV), (dict(dmul=None), INV), (dict(mul=None), INV), (dict(act=9), INV),
       (dict(udt=Q8, ue=None), INV), (dict(udt=Q8, me=None), INV), (dict(dt=F32), DTYPE), (dict(udt=F16), DTYPE), (dict(udt=F32), DTYPE),
       (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(ldu=255), SHAPE), (dict(ldm=255), SHAPE), (dict(ldo=255), SHAPE), (dict(ldd=255), SHAPE),
       (dict(U=ODD), ALIGN), (dict(U=MIS, udt=Q8), ALIGN), (dict(mul=MIS, udt=Q8), ALIGN), (dict(dU=ODD), ALIGN), (dict(dmul=ODD), ALIGN),
       (dict(db=ODD), ALIGN), (dict(ws=None), WS), (dict(short=1), WS), (dict(ws=MIS), ALIGN), (dict(M=1 << 36), UNSUP)]


@pytest.mark.parametrize("kw,status", BWD + [(dict(X=None), INV), (dict(xexps=None, xdt=Q8), INV), (dict(codes=None), INV), (dict(N=0), SHAPE),
                                             (dict(ldx=19), SHAPE), (dict(xdt=7), DTYPE), (dict(X=ODD), ALIGN), (dict(exps=MIS), ALIGN)])
def test_bwd_dx8_act(kw, status):
    a = dict(dict(X=A, xdt=BF16, xexps=A, M=70, N=20, K=256, ldx=20, codes=A, exps=A, act=2, U=A, udt=BF16, ue=A, ldu=256, mul=A, me=A, ldm=256,
                  dt=BF16, dU=A, ldo=256, dmul=A, ldd=256, db=A, ws=A, short=0), **kw)
    need = needed(slim.slim_bwd_dx8_act_workspace, a["xdt"], a["M"], a["N"], a["K"], a["dt"], 1, status=status)
    assert slim.slim_bwd_dx8_act(a["X"], a["xdt"], a["xexps"], a["M"], a["N"], a["K"], a["ldx"], a["codes"], a["exps"], a["act"], a["U"], a["udt"],
                                 a["ue"], a["ldu"], a["mul"], a["me"], a["ldm"], a["dt"], a["dU"], a["ldo"], a["dmul"], a["ldd"], a["db"], a["ws"],
                                 need - a["short"], None) == status


@pytest.mark.parametrize("kw,status", BWD + [(dict(X=None), INV), (dict(ldx=255), SHAPE), (dict(X=ODD), ALIGN), (dict(db=A + 2), ALIGN)])
def test_act_bwd(kw, status):
    a = dict(dict(X=A, M=70, K=256, ldx=256, act=2, U=A, udt=BF16, ue=A, ldu=256, mul=A, me=A, ldm=256, dt=BF16, dU=A, ldo=256, dmul=A, ldd=256,
                  db=A, ws=A, short=0), **kw)
    need = needed(slim.slim_act_bwd_workspace, a["M"], a["K"], 1, status=status)
    assert slim.slim_act_bwd(a["X"], a["dt"], a["ldx"], a["M"], a["K"], a["act"], a["U"], a["udt"], a["ue"], a["ldu"], a["mul"], a["me"], a["ldm"],
                             a["dU"], a["ldo"], a["dmul"], a["ldd"], a["db"], a["ws"], need - a["short"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(xexps=None, xdt=Q8), INV), (dict(W=None), INV), (dict(ids=None), INV), (dict(weights=None), INV),
    (dict(xdt=9), DTYPE), (dict(wdt=Q8), DTYPE), (dict(M=-1), SHAPE), (dict(K=0), SHAPE), (dict(K=WIDE, ldx=WIDE, ldw=WIDE), SHAPE),
    (dict(ldx=255), SHAPE), (dict(ldw=255), SHAPE), (dict(E=0), SHAPE), (dict(top=0), SHAPE), (dict(top=41), SHAPE), (dict(top=17), UNSUP),
    (dict(E=513), UNSUP), (dict(M=1 << 34), UNSUP), (dict(M=1 << 27), UNSUP), (dict(X=ODD), ALIGN), (dict(X=MIS, xdt=Q8), ALIGN), (dict(W=A + 2), ALIGN),
    (dict(ids=A + 2), ALIGN), (dict(weights=A + 2), ALIGN), (dict(ws=None), WS), (dict(short=1), WS), (dict(ws=MIS), ALIGN),
    (dict(M=0, X=None), OK)])
def test_route(kw, status):
    a = dict(dict(X=A, xdt=BF16, xexps=A, M=3, K=256, ldx=256, W=A, wdt=F32, E=40, ldw=256, top=4, ids=A, weights=A, ws=A, short=0), **kw)
    need = needed(slim.slim_route_workspace, a["M"], a["E"], a["K"], status=status)
    assert slim.slim_route(a["X"], a["xdt"], a["xexps"], a["M"], a["K"], a["ldx"], a["W"], a["wdt"], a["E"], a["ldw"], a["top"], 1, a["ids"],
                           a["weights"], a["ws"], need - a["short"], None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(X=None), INV), (dict(xexps=None, xdt=Q8), INV), (dict(g=None), INV), (dict(ge=None), INV), (dict(u=None), INV), (dict(ue=None), INV),
    (dict(d=None), INV), (dict(de=None), INV), (dict(ids=None), INV), (dict(weights=None), INV), (dict(Y=None), INV), (dict(act=5), INV),
    (dict(xdt=F32), DTYPE), (dict(dt=F32), DTYPE), (dict(dt=Q8), DTYPE), (dict(M=-1), SHAPE), (dict(D=0), SHAPE), (dict(F=0), SHAPE),
    (dict(E=0), SHAPE), (dict(top=0), SHAPE), (dict(D=WIDE, ldx=WIDE, ldy=WIDE, ldr=WIDE), SHAPE), (dict(ldx=255), SHAPE), (dict(ldy=255), SHAPE),
    (dict(ldr=255), SHAPE), (dict(M=65), UNSUP), (dict(E=513), UNSUP), (dict(top=17), UNSUP), (dict(X=ODD), ALIGN), (dict(X=MIS, xdt=Q8), ALIGN),
    (dict(g=MIS), ALIGN), (dict(ue=MIS), ALIGN), (dict(de=MIS), ALIGN), (dict(ids=A + 2), ALIGN), (dict(weights=A + 2), ALIGN), (dict(res=ODD), ALIGN),
    (dict(Y=ODD), ALIGN), (dict(ws=None), WS), (dict(short=1), WS), (dict(ws=MIS), ALIGN), (dict(M=0, X=None), OK)])
def test_moe8(kw, status):
    a = dict(dict(X=A, xdt=BF16, xexps=A, M=7, D=256, ldx=256, F=300, E=40, g=A, ge=A, u=A, ue=A, d=A, de=A, act=4, ids=A, weights=A, top=4, res=A,
                  ldr=256, Y=A, dt=BF16, ldy=256, ws=A, short=0), **kw)
    need = needed(slim.slim_moe8_workspace, a["M"], a["D"], a["F"], a["E"], a["top"], status=status)
    assert slim.slim_moe8(a["X"], a["xdt"], a["xexps"], a["M"], a["D"], a["ldx"], a["F"], a["E"], a["g"], a["ge"], a["u"], a["ue"], a["d"], a["de"],
                          a["act"], a["ids"], a["weights"], a["top"], a["res"], a["ldr"], a["Y"], a["dt"], a["ldy"], a["ws"], need - a["short"],
                          None) == status


def test_the_largest_that_are_taken():
    slim.slim_linear8_act_workspace(Q8, 1 << 14, 1 << 22, 28672, F16, 0)
    slim.slim_act_bwd_workspace(1 << 20, 28672, 1)
    assert slim.slim_moe8_workspace(64, 8192, 28672, 512, 16) > 0
    assert slim.slim_moe8_workspace(0, 8192, 28672, 512, 16) == slim.slim_linear8_act_workspace(F16, 0, 10, 10, F16, 1) == 0
    # a row's codes are turned up in the product's own launch
    assert slim.slim_linear8_act_workspace(BF16, 1, 4096, 4096, BF16, 0) == 0
    # one block's sums over rows are the result
    assert slim.slim_act_bwd_workspace(16, 4096, 1) == 0 and slim.slim_act_bwd_workspace(17, 4096, 1) > 0


gpu = lambda *s, dt=torch.bfloat16: torch.zeros(s, dtype=dt).as_subclass(OnGpu)


def rows8(m, k):
    return {"codes": gpu(m, -(-k // 128) * 128, dt=torch.uint8), "exps": gpu(m, -(-k // 512) * 4, dt=torch.uint8), "M": m, "K": k}


def weight8(n, k):
    w = lambda n, k: (gpu(-(-n // 16), -(-k // 128), 2, 4, 16, 16, dt=torch.uint8), gpu(-(-n // 128), -(-k // 512) * 4, dt=torch.uint8))
    (c, e), (ct, et) = w(n, k), w(k, n)
    return {"codes": c, "exps": e, "codesT": ct, "expsT": et, "N": n, "K": k}


def experts8(e, n, k):
    return {"codes": gpu(e, -(-n // 16), -(-k // 128), 2, 4, 16, 16, dt=torch.uint8), "exps": gpu(e, -(-n // 128), -(-k // 512) * 4, dt=torch.uint8),
            "E": e, "N": n, "K": k}


def test_binding_refuses_what_does_not_fit(monkeypatch):
    monkeypatch.setattr(slim, "_stream_on", lambda dev: 0)
    x, p, u = gpu(4, 256), weight8(32, 256), gpu(4, 32)
    bad = [
        lambda: slim.linear8_act(x, p, act="tanh"), lambda: slim.linear8_act(x, p, act=2), lambda: slim.linear8_act(gpu(4, 255), p),
        lambda: slim.linear8_act(x, p, bias=gpu(31)), lambda: slim.linear8_act(x, p, mul=gpu(4, 31)), lambda: slim.linear8_act(x, p, mul=gpu(3, 32)),
        lambda: slim.linear8_act(x, p, mul=u, residual=gpu(4, 32, dt=torch.float16)), lambda: slim.linear8_act(x, p, out=gpu(4, 33)),
        lambda: slim.linear8_act(x, p, q8=True, out=rows8(4, 31)), lambda: slim.linear8_act(torch.zeros(4, 256), p),
        lambda: slim.linear8_act(x, p, residual=u.expand(1, 4, 32)), lambda: slim.linear8_act(x, p, mul=gpu(1, 32).expand(4, 32)),
        lambda: slim.bwd_dx8_act(u, p, gpu(4, 255), act="gelu"), lambda: slim.bwd_dx8_act(x, p, x, act="gelu"),
        lambda: slim.bwd_dx8_act(u, p, rows8(4, 255), act="gelu"), lambda: slim.bwd_dx8_act(u, p, x, act="gelu", mul=gpu(5, 256)),
        lambda: slim.act_bwd(x, gpu(4, 255), act="gelu"), lambda: slim.act_bwd(x, x, act="gelu", mul=gpu(4, 256, dt=torch.float16)),
        lambda: slim.act_bwd(x, x, act="gelu", out=gpu(4, 256, dt=torch.float16)), lambda: slim.act_bwd(torch.zeros(4, 256), x),
        lambda: slim.route(x, gpu(8, 255), 2), lambda: slim.route(x, gpu(8, 256), 9), lambda: slim.route(x, gpu(8, 256), 0),
        lambda: slim.route(x, torch.zeros(8, 256), 2)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: slim.act_bwd(x, rows8(4, 256), act="gelu", mul=x), lambda: slim.act_bwd(x, x, act="gelu", mul=rows8(4, 256)),
                 lambda: slim.linear8_act(x, p, bias=gpu(32, dt=torch.int32)), lambda: slim.linear8_act(gpu(4, 256, dt=torch.int16), p),
                 lambda: slim.route(x, gpu(8, 256, dt=torch.int8), 2)):
        with pytest.raises(TypeError):
            call()
    # a type that the library does not take for results
    with pytest.raises(slim.SlimError):
        slim.linear8_act(x, p, dtype=torch.float32)
    with pytest.raises(slim.SlimError):
        slim.act_bwd(gpu(4, 256, dt=torch.float32), gpu(4, 256, dt=torch.float32), act="gelu")


def test_binding_refuses_experts_that_do_not_fit(monkeypatch):
    monkeypatch.setattr(slim, "_stream_on", lambda dev: 0)
    x, g, d = gpu(4, 256), experts8(6, 300, 256), experts8(6, 256, 300)
    ids, w = gpu(4, 2, dt=torch.int32), gpu(4, 2, dt=torch.float32)
    for call in (lambda: slim.moe8(gpu(4, 255), g, g, d, ids, w), lambda: slim.moe8(x, g, experts8(6, 299, 256), d, ids, w),
                 lambda: slim.moe8(x, g, experts8(5, 300, 256), d, ids, w), lambda: slim.moe8(x, g, g, g, ids, w),
                 lambda: slim.moe8(x, dict(g, codes=g["codes"][:5]), g, d, ids, w), lambda: slim.moe8(x, dict(g, exps=g["exps"][:, :2]), g, d, ids, w),
                 lambda: slim.moe8(x, g, g, d, ids[:3], w), lambda: slim.moe8(x, g, g, d, ids, w[:, :1]), lambda: slim.moe8(x, g, g, d, ids[:3], w[:3]),
                 lambda: slim.moe8(x, g, g, d, ids.t().contiguous().t(), w), lambda: slim.moe8(x, g, g, d, ids, w, act="swish"),
                 lambda: slim.moe8(x, g, g, d, ids, w, residual=gpu(4, 255)), lambda: slim.moe8(x, g, g, d, ids, w, out=gpu(3, 256)),
                 lambda: slim.moe8(x, g, g, d, torch.zeros((4, 2), dtype=torch.int32), w), lambda: slim.pack8_experts(gpu(4, 4)), lambda: slim.pack8_experts(gpu(0, 4, 4))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: slim.moe8(x, g, g, d, ids.long(), w), lambda: slim.moe8(x, g, g, d, ids, w.bfloat16()),
                 lambda: slim.moe8(x, dict(g, codes=g["codes"].short()), g, d, ids, w)):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(slim.SlimError) as e:
        slim.moe8(gpu(65, 256), g, g, d, gpu(65, 2, dt=torch.int32), gpu(65, 2, dt=torch.float32))
    assert e.value.status == UNSUP
