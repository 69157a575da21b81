"""slim_norm and slim_norm_bwd against the oracle in 64 bits.

Bounds, with v = 2^-24 and u the last half place of the result's type (2^-24, 2^-11, 2^-8): fp32 sums of a row go through
chains of at most 40 additions (a thread's own, the wave's, the block's), so the mean is within 40 v mean|x|, the relative
error of rstd within 40 v + that of the deviations; y and dx within u |result| + 64 v of the terms that make it up. Column
sums over M rows: (M + 64) v of the sum of magnitudes."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim, synth
from tests.gpu_common import dev, host

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11, "fp32": 2.0 ** -24}
V = 2.0 ** -24
EPS = 1e-5


def inputs(m, k, dtype, params="fp32", seed=0):
    rng = synth.stream(seed, f"norm/{m}x{k}/{dtype}")
    x = rng.standard_normal((m, k)) * 10.0 ** rng.uniform(-2, 2, (m, 1)) + rng.uniform(-3, 3, (m, 1))
    x *= np.where(rng.random(k) < 0.01, 20.0, 1.0)
    t = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    g = torch.from_numpy((1 + 0.3 * rng.standard_normal(k)).astype(np.float32)).to(DT[params])
    b = torch.from_numpy((0.3 * rng.standard_normal(k)).astype(np.float32)).to(DT[params])
    return t, g, b


def f64(t):
    return t.double().cpu().numpy()


def check_forward(t, g, b, rms, y, mean, rstd, u, y_ref=None):
    x, g, b = f64(t), None if g is None else f64(g), None if b is None else f64(b)
    ref, mu, rs = act8.norm(x, g, b, EPS, rms)
    ax = np.abs(x).mean(1)
    if rms:
        assert mean is None
    else:
        assert np.all(np.abs(f64(mean) - mu) <= 40 * V * ax)
    # a relative error d of the deviations' scale moves rstd by d at most
    dev_err = 80 * V * (1 + (0 if rms else 1) * ax * rs)
    assert np.all(np.abs(f64(rstd) - rs) <= dev_err * rs)
    gg = 1.0 if g is None else np.abs(g)
    terms = ((np.abs(x) + ax[:, None]) * rs[:, None] * gg + np.abs(ref)) * (1 + (ax * rs)[:, None])
    lim = u * np.abs(ref) + 128 * V * terms + (2.0 ** -25 if u == 2.0 ** -11 else 0.0)
    assert np.all(np.abs(y - ref) <= lim)


WIDTHS = [1, 7, 8, 100, 512, 513, 1000, 1024, 1025, 2048, 4096, 4097, 5120, 8192, 8193, 12288, 16384, 16392, 28672, 40001]


@pytest.mark.parametrize("k", WIDTHS)
@pytest.mark.parametrize("dtype,params", [("bf16", "fp32"), ("fp16", "fp16"), ("fp32", "fp32")])
@pytest.mark.parametrize("rms", [False, True])
def test_forward(k, dtype, params, rms):
    m = 3 if k > 4096 else 9
    print(f"norm m={m} k={k} {dtype} rms={rms}", flush=True)
    t, g, b = inputs(m, k, dtype, params)
    b = None if rms else b
    y, mean, rstd = slim.norm(t.cuda(), g.cuda(), None if rms else b.cuda(), eps=EPS, rms=rms)
    assert y.dtype == DT[dtype]
    check_forward(t, g, b, rms, f64(y), mean, rstd, U[dtype])


@pytest.mark.parametrize("m,k", [(1, 4096), (5, 1), (700, 64), (3000, 520), (2500, 1024), (1500, 4096), (1100, 5000), (300, 16384)])
def test_forward_many_rows(m, k):
    # more rows than blocks: gamma and beta are held, the next row is loaded ahead
    print(f"norm m={m} k={k}", flush=True)
    t, g, b = inputs(m, k, "bf16", "bf16", seed=1)
    y, mean, rstd = slim.norm(t.cuda(), g.cuda(), b.cuda(), eps=EPS)
    check_forward(t, g, b, False, f64(y), mean, rstd, U["bf16"])


@pytest.mark.parametrize("m,k", [(1, 4096), (3, 1), (9, 100), (700, 128), (5, 129), (1300, 1000), (7, 4096), (6, 5000), (600, 8192), (3, 12288), (2, 28680),
                                 (2, 40001)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rms", [False, True])
def test_result_in_8_bits(m, k, dtype, rms):
    print(f"norm q8 m={m} k={k} {dtype} rms={rms}", flush=True)
    t, g, b = inputs(m, k, dtype, seed=2)
    b = None if rms else b.cuda()
    q, mean, rstd = slim.norm(t.cuda(), g.cuda(), b, eps=EPS, rms=rms, q8=True)
    # to the bit what quant8 makes of the same fp32 results, which an fp32 input gives
    y, mean32, rstd32 = slim.norm(t.float().cuda(), g.cuda(), b, eps=EPS, rms=rms)
    want = slim.quant8(y)
    assert torch.equal(rstd, rstd32) and (rms or torch.equal(mean, mean32))
    assert torch.equal(q["exps"], want["exps"]) and torch.equal(q["codes"], want["codes"])


def test_plain_rows_without_parameters():
    t, _, _ = inputs(5, 300, "fp32", seed=3)
    y, mean, rstd = slim.norm(t.cuda())
    check_forward(t, None, None, False, f64(y), mean, rstd, U["fp32"])


def test_rows_far_from_zero_keep_their_variance():
    # deviations 1e-3 of the mean: a variance taken as E x^2 - mu^2 would lose all but a few bits
    rng = synth.stream(4, "norm/far")
    x = torch.from_numpy((1000.0 + rng.standard_normal((6, 5000))).astype(np.float32))
    y, mean, rstd = slim.norm(x.cuda(), eps=0.0)
    ref, mu, rs = act8.norm(f64(x), None, None, 0.0, False)
    assert np.all(np.abs(f64(rstd) / rs - 1) < 1e-5) and np.all(np.abs(f64(mean) - mu) <= 40 * V * 1000)


def test_constant_and_zero_rows():
    x = torch.zeros((3, 777), dtype=torch.float32)
    x[1] = 5.0
    y, mean, rstd = slim.norm(x.cuda(), eps=EPS)
    assert bool((y == 0).all()) and host(mean).tolist() == [0.0, 5.0, 0.0]
    assert np.allclose(host(rstd), EPS ** -0.5, rtol=1e-6)


def test_nan_and_infinite_rows_stay_apart():
    t, g, b = inputs(700, 1000, "bf16", seed=5)
    clean = slim.norm(t.cuda(), g.cuda(), b.cuda())[0]
    t[3, 7], t[650, 999] = float("nan"), float("inf")
    y = slim.norm(t.cuda(), g.cuda(), b.cuda())[0]
    rows = torch.ones(700, dtype=torch.bool)
    rows[[3, 650]] = False
    assert bool(y[3].isnan().all()) and bool(y[650].isnan().any()) and torch.equal(y[rows.cuda()], clean[rows.cuda()])


@pytest.mark.parametrize("q8", [False, True])
def test_strides_and_the_bytes_around_the_result(q8):
    t, g, b = inputs(12, 700, "fp16", seed=6)
    view = t.cuda()[1:10, 3:3 + 601]
    y, mean, rstd = slim.norm(view, g.cuda()[:601], b.cuda()[:601], q8=q8)
    plain, *_ = slim.norm(view.contiguous(), g.cuda()[:601], b.cuda()[:601], q8=q8)
    if q8:
        assert torch.equal(y["codes"], plain["codes"]) and torch.equal(y["exps"], plain["exps"])
        return
    assert torch.equal(y, plain)
    buf = torch.full((11, 640), -7.0, dtype=torch.float16, device="cuda")
    slim.norm(view, g.cuda()[:601], b.cuda()[:601], out=buf[1:10, 5:606])
    assert torch.equal(buf[1:10, 5:606], plain)
    buf[1:10, 5:606] = -7.0
    assert bool((buf == -7).all())


# ------------------------------------------------------------------------------------- backward
def check_backward(dy, x, g, mean, rstd, rms, dx, dg, db, u):
    """x: the float64 rows that the kernel reads (a checkpoint's values, where it is one)."""
    m, k = dy.shape
    mu, rs = np.zeros(m) if rms else f64(mean), f64(rstd)
    rdx, rdg, rdb = act8.norm_bwd(dy, x, g, mu, rs, rms)
    xm = (np.abs(x) + np.abs(mu)[:, None]) * rs[:, None]            # |xh| before its difference
    t = np.abs(dy) * (1.0 if g is None else np.abs(g))
    terms = rs[:, None] * (t + t.mean(1, keepdims=True) + xm * (t * xm).mean(1, keepdims=True))
    lim = u * np.abs(rdx) + 64 * V * terms + (2.0 ** -25 if u == 2.0 ** -11 else 0.0)
    assert np.all(np.abs(f64(dx) - rdx) <= lim)
    assert np.all(np.abs(f64(dg) - rdg) <= (m + 64) * V * (np.abs(dy) * xm).sum(0) + 1e-30)
    if rms:
        assert db is None
    else:
        assert np.all(np.abs(f64(db) - rdb) <= (m + 64) * V * np.abs(dy).sum(0) + 1e-30)


@pytest.mark.parametrize("m,k", [(1, 1), (1, 4096), (3, 7), (9, 100), (2100, 64), (333, 1000), (40, 1024), (3, 1025), (900, 2048), (5, 4097), (700, 5120),
                                 (530, 8192), (3, 8193), (5, 12288), (4, 16384), (300, 16392), (3, 28672)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rms,q8", [(False, False), (False, True), (True, False), (True, True)])
def test_backward(m, k, dtype, rms, q8):
    print(f"norm_bwd m={m} k={k} {dtype} rms={rms} q8={q8}", flush=True)
    t, g, b = inputs(m, k, dtype, "fp32", seed=7)
    dy = torch.from_numpy(synth.stream(8, f"norm/dy/{m}x{k}").standard_normal((m, k)).astype(np.float32)).to(DT[dtype])
    x = t.cuda()
    _, mean, rstd = slim.norm(x, g.cuda(), None if rms else b.cuda(), rms=rms)
    if q8:
        x = slim.quant8(x)
        xv = act8.values_rows(host(x["codes"]), host(x["exps"]), k)
    else:
        xv = f64(t)
    dx, dg, db = slim.norm_bwd(dy.cuda(), x, g.cuda(), mean, rstd)
    assert dx.dtype == DT[dtype] and dg.dtype == torch.float32
    check_backward(f64(dy), xv, f64(g), mean, rstd, rms, dx, dg, db, U[dtype])


@pytest.mark.parametrize("m,k", [(600, 5001), (300, 8191), (5, 12287), (300, 16383), (3, 28671)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("q8", [False, True])
def test_rows_that_end_inside_a_vector(m, k, dtype, q8):
    print(f"norm and norm_bwd m={m} k={k} {dtype} q8={q8}", flush=True)
    t, g, b = inputs(m, k, dtype, "fp32", seed=9)
    y, mean, rstd = slim.norm(t.cuda(), g.cuda(), b.cuda())
    check_forward(t, g, b, False, f64(y), mean, rstd, U[dtype])
    dy = torch.from_numpy(synth.stream(10, f"norm/dy/{m}x{k}").standard_normal((m, k)).astype(np.float32)).to(DT[dtype])
    x = slim.quant8(t.cuda()) if q8 else t.cuda()
    xv = act8.values_rows(host(x["codes"]), host(x["exps"]), k) if q8 else f64(t)
    dx, dg, db = slim.norm_bwd(dy.cuda(), x, g.cuda(), mean, rstd)
    check_backward(f64(dy), xv, f64(g), mean, rstd, False, dx, dg, db, U[dtype])


@pytest.mark.parametrize("rms", [False, True])
def test_backward_against_differences(rms):
    # the kernel's gradients against differences of the 64-bit forward
    rng = synth.stream(9, "norm/diff")
    x, dy, g, b = rng.standard_normal((6, 37)), rng.standard_normal((6, 37)), 1 + 0.2 * rng.standard_normal(37), rng.standard_normal(37)
    x, dy, g, b = (a.astype(np.float32) for a in (x, dy, g, b))
    _, mean, rstd = slim.norm(dev(x), dev(g), None if rms else dev(b), rms=rms)
    dx, dg, db = slim.norm_bwd(dev(dy), dev(x), dev(g), mean, rstd)
    loss = lambda x, g, b: (act8.norm(x, g, None if rms else b, EPS, rms)[0] * dy).sum()
    args = [a.astype(np.float64) for a in (x, g, b)]
    for at, grad in ((0, dx), (1, dg)) + (() if rms else ((2, db),)):
        d = rng.standard_normal(args[at].shape)
        hi, lo = list(args), list(args)
        hi[at], lo[at] = args[at] + 1e-6 * d, args[at] - 1e-6 * d
        want = (loss(*hi) - loss(*lo)) / 2e-6
        # differences to 1e-8; fp32 gradients to 64 v of their terms (at most about 10 each, 222 of them)
        assert abs(want - (f64(grad) * d).sum()) < 1e-6 + 64 * V * 10 * 222


@pytest.mark.parametrize("k", [100, 4096, 12288, 20000])
def test_backward_of_rows_far_from_zero(k):
    # fp32 rows about 1000 with deviations of 1: xh is (x - mean) rstd with the difference taken first, exact but for the mean's
    # own rounding (2^-25 of it) and a rounding each, so off by (1000 + 4 |xh|) 2^-24 at most
    rng = synth.stream(13, f"norm/far/{k}")
    x = (1000 + rng.standard_normal((4, k))).astype(np.float32)
    dy = rng.standard_normal((4, k)).astype(np.float32)
    _, mean, rstd = slim.norm(dev(x))
    dg = f64(slim.norm_bwd(dev(dy), dev(x), None, mean, rstd)[1])
    mu, rs = x.astype(np.float64).mean(1, keepdims=True), f64(rstd)[:, None]
    xh = (x.astype(np.float64) - f64(mean)[:, None]) * rs
    assert np.all(np.abs(f64(mean)[:, None] - mu) <= 40 * V * 1010)
    assert np.all(np.abs(dg - (dy * xh).sum(0)) <= V * (np.abs(dy) * (8 * np.abs(xh))).sum(0) + 8 * V * np.abs(dy * xh).sum(0))


def test_backward_in_place_and_strided():
    for k in (601, 9000):
        t, g, b = inputs(12, 2 * k, "bf16", seed=10)
        x, dy = t.cuda()[1:10, 3:3 + k], t.cuda()[2:11, k:2 * k]
        _, mean, rstd = slim.norm(x, g.cuda()[:k], b.cuda()[:k])
        want = slim.norm_bwd(dy.contiguous(), x.contiguous(), g.cuda()[:k], mean, rstd)
        got = slim.norm_bwd(dy, x, g.cuda()[:k], mean, rstd)
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        buf = torch.full((11, k + 10), -7.0, dtype=torch.bfloat16, device="cuda")
        buf[1:10, 5:5 + k] = dy
        over = slim.norm_bwd(buf[1:10, 5:5 + k], x, g.cuda()[:k], mean, rstd, out=buf[1:10, 5:5 + k])
        assert all(torch.equal(a, b) for a, b in zip(over, want))
        buf[1:10, 5:5 + k] = -7.0
        assert bool((buf == -7).all())


def test_no_rows():
    e = torch.empty((0, 50), dtype=torch.bfloat16, device="cuda")
    y, mean, rstd = slim.norm(e)
    assert y.shape == (0, 50) and rstd.shape == (0,)
    dx, dg, db = slim.norm_bwd(e, e, None, mean, rstd)
    assert dx.shape == (0, 50) and bool((dg == 0).all()) and bool((db == 0).all())


def test_another_stream_and_repeats():
    t, g, b = inputs(900, 1000, "fp16", seed=11)
    x = t.cuda()
    y, mean, rstd = slim.norm(x, g.cuda(), b.cuda())
    first = slim.norm_bwd(y, x, g.cuda(), mean, rstd)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        for _ in range(3):
            again = slim.norm_bwd(y, x, g.cuda(), mean, rstd)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(again, first))


@pytest.mark.parametrize("k", [100, 1000, 1025, 4097, 5120, 12289, 20000, 28680, 40001])
@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("fp16", False), ("fp32", False), ("bf16", True), ("fp16", True)])
def test_rows_of_one_value_far_from_zero(k, dtype, q8):
    # 13 * 4096: exact in every type, in 8 bits too, and so is its sum over a row (13 k < 2^24). Then the mean is the value and
    # xh is zero exactly, while rstd = 316 would make 0.5 of a rounding step of mean * rstd
    value = 13 * 4096.0
    t = torch.full((5, k), value, dtype=DT[dtype], device="cuda")
    rng = synth.stream(14, f"norm/one/{k}")
    b = dev((0.3 * rng.standard_normal(k)).astype(np.float32))
    dy = torch.from_numpy(rng.standard_normal((5, k)).astype(np.float32)).to(DT[dtype]).cuda()
    y, mean, rstd = slim.norm(t, None, b)
    assert bool((mean == value).all()) and torch.equal(y, b.to(DT[dtype]).expand(5, k))
    _, dg, db = slim.norm_bwd(dy, slim.quant8(t) if q8 else t, None, mean, rstd)
    assert bool((dg == 0).all())
    assert np.all(np.abs(f64(db) - f64(dy).sum(0)) <= 69 * V * np.abs(f64(dy)).sum(0))
