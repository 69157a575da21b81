"""slim_grad_w8 against the 64-bit product of dY and the checkpoint's values: |fp32 sum - exact| <= 2 M 2^-24 sum|products|
for any order of an M-term fp32 sum of exact products."""
import numpy as np
import pytest
import torch

from oracle import act8, slope_train
from paper_2608_24070_amd import slim, synth
from tests.gpu_common import dev, host

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def inputs(m, n, k, dtype, seed=0):
    rng = synth.stream(seed, f"grad_w8/{m}x{n}x{k}/{dtype}")
    dy = torch.from_numpy((rng.standard_normal((m, n)) * 0.01).astype(np.float32)).to(DT[dtype])
    x = rng.standard_normal((m, k)) * 4.0 ** rng.integers(-2, 3, (m, 1))
    x = torch.from_numpy((x * np.where(rng.random(k) < 0.01, 20.0, 1.0)).astype(np.float32)).to(DT[dtype])
    return dy, x


def check(got, dy, x, pick=lambda a: a):
    ref, mag = pick(dy.T @ x), pick(np.abs(dy).T @ np.abs(x))
    assert np.all(np.abs(host(got) - ref) <= 2.0 * dy.shape[0] * 2.0 ** -24 * mag + 1e-30)


def kept(n, k, seed=0):
    w = synth.stream(seed, f"grad_w8/w/{n}x{k}").standard_normal((n, k)).astype(np.float32)
    p = slim.pack16(dev(w))
    mask = slope_train.pack16(w)["mask"].astype(bool)
    return p, lambda a: a[mask].reshape(n, k // 2)


SIZES = [(1, 1, 1), (1, 128, 128), (5, 3, 130), (31, 200, 64), (32, 128, 256), (33, 129, 127), (200, 300, 500), (999, 515, 768), (1500, 256, 256),
         (2049, 40, 300), (64, 1030, 520)]


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_whole_gradient(m, n, k, dtype):
    print(f"grad_w8 m={m} n={n} k={k} {dtype}", flush=True)
    dy, x = inputs(m, n, k, dtype)
    q = slim.quant8(x.cuda())
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    check(slim.grad_w8(dy.cuda(), q), dy.double().numpy(), xv)


@pytest.mark.parametrize("m,n,k", [(1, 16, 16), (37, 256, 384), (200, 100, 144), (1000, 384, 512), (64, 515, 640), (3000, 256, 272)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_kept_positions(m, n, k, dtype):
    print(f"grad_w8 kept m={m} n={n} k={k} {dtype}", flush=True)
    dy, x = inputs(m, n, k, dtype, seed=1)
    p, pick = kept(n, k)
    q = slim.quant8(x.cuda())
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    check(slim.grad_w8(dy.cuda(), q, p), dy.double().numpy(), xv, pick)


# layers of 128 and more tiles of 256 x 256; odd widths end inside a word, a tile and a group
WIDE = [(1, 8200, 1024), (70, 8191, 1021), (33, 8250, 1000), (129, 2100, 4000)]


@pytest.mark.parametrize("m,n,k", WIDE)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_large_layers(m, n, k, dtype):
    print(f"grad_w8 wide m={m} n={n} k={k} {dtype}", flush=True)
    dy, x = inputs(m, n, k, dtype, seed=8)
    q = slim.quant8(x.cuda())
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    got = slim.grad_w8(dy.cuda(), q)
    check(got, dy.double().numpy(), xv)
    # rows that are aligned, as part of wider ones that NaN fills, and rows that start anywhere: the same bits
    for start, width in ((8, n + 24 - n % 8), (3, n + 7)):
        buf = torch.full((m, width), float("nan"), dtype=DT[dtype], device="cuda")
        buf[:, start:start + n] = dy.cuda()
        assert torch.equal(slim.grad_w8(buf[:, start:start + n], q), got), start


@pytest.mark.parametrize("m,n,k", [(45, 16387, 512), (100, 4096, 2064)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_large_layers_kept_positions(m, n, k, dtype):
    print(f"grad_w8 wide kept m={m} n={n} k={k} {dtype}", flush=True)
    dy, x = inputs(m, n, k, dtype, seed=9)
    p, pick = kept(n, k)
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    check(slim.grad_w8(dy.cuda(), slim.quant8(x.cuda()), p), dy.double().numpy(), xv, pick)


def test_large_layer_of_no_rows():
    q = slim.quant8(torch.empty((0, 1024), dtype=torch.bfloat16, device="cuda"))
    g = slim.grad_w8(torch.empty((0, 8200), dtype=torch.bfloat16, device="cuda"), q)
    assert g.shape == (8200, 1024) and bool((g == 0).all())


# 128 x 128 tiles that fill the chip, over one slice of the rows and over three, then 256 x 256 tiles: whole rounds of them, one
# round not quite full, and rounds that leave most of the last idle
MANY = [(520, 2000, 1040), (513, 2051, 1030), (3000, 1000, 1040), (2999, 1003, 1041), (255, 4097, 4112),
        (97, 4096, 4090), (200, 8192, 2048), (131, 3961, 3888), (1537, 2301, 4352), (769, 4099, 2549), (800, 4352, 4096)]


@pytest.mark.parametrize("m,n,k", MANY)
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_many_tiles(m, n, k, dtype):
    print(f"grad_w8 many tiles m={m} n={n} k={k} {dtype}", flush=True)
    dy, x = inputs(m, n, k, dtype, seed=11)
    q = slim.quant8(x.cuda())
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    got = slim.grad_w8(dy.cuda(), q)
    check(got, dy.double().numpy(), xv)
    if k % 16 == 0:
        p, pick = kept(n, k)
        assert np.array_equal(host(slim.grad_w8(dy.cuda(), q, p)), pick(host(got)))
    # rows that are aligned, as part of wider ones that NaN fills, and rows that start anywhere: the same bits
    for start, width in ((8, n + 24 - n % 8), (3, n + 7)):
        buf = torch.full((m, width), float("nan"), dtype=DT[dtype], device="cuda")
        buf[:, start:start + n] = dy.cuda()
        assert torch.equal(slim.grad_w8(buf[:, start:start + n], q), got), start


@pytest.mark.parametrize("n", [1, 7, 15, 16, 17, 130])
def test_narrow_layers_over_many_rows(n):
    # slices of the rows, joined; rows shorter than a load
    dy, x = inputs(2600, n, 140, "bf16", seed=10)
    q = slim.quant8(x.cuda())
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), 140)
    buf = torch.full((2600, n + 5), float("nan"), dtype=torch.bfloat16, device="cuda")
    buf[:, 3:3 + n] = dy.cuda()
    got = slim.grad_w8(dy.cuda(), q)
    check(got, dy.double().numpy(), xv)
    assert torch.equal(slim.grad_w8(buf[:, 3:3 + n], q), got)


@pytest.mark.parametrize("m,n,k", [(50, 130, 300), (700, 300, 260), (2000, 520, 640)])
def test_small_integers_are_exact(m, n, k):
    rng = synth.stream(2, f"grad_w8/int/{m}x{n}x{k}")
    dy, x = rng.integers(-3, 4, (m, n)), rng.integers(-4, 5, (m, k))
    for dt in (torch.float16, torch.bfloat16):
        g = slim.grad_w8(dev(dy.astype(np.float32)).to(dt), slim.quant8(dev(x.astype(np.float32)).to(dt)))
        assert np.array_equal(host(g).astype(int), dy.T @ x)


def test_same_as_the_16_bit_gradient_of_the_same_values():
    dy, x = inputs(300, 256, 384, "bf16", seed=3)
    p, _ = kept(256, 384)
    q = slim.quant8(x.cuda())
    a, b = host(slim.grad_w8(dy.cuda(), q, p)), host(slim.grad_w(dy.cuda(), slim.dequant8(q, torch.bfloat16), p))
    assert np.linalg.norm(a - b) <= 1e-6 * np.linalg.norm(b)


@pytest.mark.parametrize("scale", [1e-30, 1e-6, 1e6, 1e30])
def test_checkpoints_of_any_size_in_bf16(scale):
    dy, x = inputs(150, 140, 200, "bf16", seed=4)
    x = (x.float() * scale).to(torch.bfloat16)
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), 200)
    check(slim.grad_w8(dy.cuda(), slim.quant8(x.cuda())), dy.double().numpy(), xv)


def test_smallest_fp16_values_are_exact():
    # fp16 subnormals as activations and as gradients
    rng = synth.stream(5, "grad_w8/sub")
    x = torch.from_numpy((rng.integers(-40, 41, (64, 128)) * 2.0 ** -24).astype(np.float32)).to(torch.float16)
    dy = torch.from_numpy((rng.integers(-40, 41, (64, 32)) * 2.0 ** -24).astype(np.float32)).to(torch.float16)
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), 128)
    check(slim.grad_w8(dy.cuda(), slim.quant8(x.cuda())), dy.double().numpy(), xv)


def test_strided_gradient_rows():
    dy, x = inputs(100, 500, 300, "bf16", seed=6)
    q = slim.quant8(x.cuda())
    view = dy.cuda()[:, 7:7 + 333]
    assert torch.equal(slim.grad_w8(view, q), slim.grad_w8(view.contiguous(), q))


def test_no_rows_gives_zeros():
    q = slim.quant8(torch.empty((0, 200), dtype=torch.bfloat16, device="cuda"))
    g = slim.grad_w8(torch.empty((0, 30), dtype=torch.bfloat16, device="cuda"), q)
    assert g.shape == (30, 200) and bool((g == 0).all())


def test_repeats_and_another_stream():
    dy, x = inputs(3000, 300, 260, "fp16", seed=7)
    q, dy = slim.quant8(x.cuda()), dy.cuda()
    first = slim.grad_w8(dy, q)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        again = slim.grad_w8(dy, q)
    s.synchronize()
    assert torch.equal(again, first) and torch.equal(slim.grad_w8(dy, q), first)
