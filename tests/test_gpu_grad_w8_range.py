"""slim_grad_w8 with fp16 dY and checkpoints past fp16's range, against the 64-bit product.

Bound: 2 M 2^-24 sum|products| for any order of an M-term fp32 sum, and what widening X to fp16 rounds off: half of fp16's
smallest step, 2^-25, or where a group of 128 columns passes 448 2^7 and is scaled down by a power of two, 2^-25 times that
power, which is less than 2^-14 of the group's largest value over the rows."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim, synth
from tests.gpu_common import dev, host
from tests.test_gpu_grad_w8 import kept

pytestmark = pytest.mark.gpu


def check(got, dy, xv, pick=lambda a: a):
    m, k = xv.shape
    top = np.abs(np.pad(xv, ((0, 0), (0, -k % 128)))).reshape(m, -1, 128).max((0, 2)).repeat(128)[:k]
    ref, mag = dy.T @ xv, np.abs(dy).T @ np.abs(xv)
    lim = 2.0 * m * 2.0 ** -24 * mag + np.abs(dy).sum(0)[:, None] * (2.0 ** -25 + 2.0 ** -39 * top) + 1e-30
    g = host(got).astype(np.float64)
    assert np.all(np.isfinite(g)) and np.all(np.abs(g - pick(ref)) <= pick(lim))


# whole tiles of 64 x 128 and 128 x 128, some over slices of the rows, and of 256 x 256
SIZES = [(5, 3, 130), (64, 200, 300), (700, 300, 500), (2600, 40, 300), (129, 2100, 4000), (70, 8191, 1021), (1537, 2301, 4352)]


def gradients(m, n, seed):
    rng = synth.stream(seed, f"grad_w8/range/{m}x{n}")
    return torch.from_numpy((rng.standard_normal((m, n)) * 0.01).astype(np.float32)).half()


@pytest.mark.parametrize("m,n,k", SIZES)
def test_the_largest_fp16_activations(m, n, k):
    # past 63488 the nearest code is 256 2^8 = 65536, which fp16 does not hold
    print(f"grad_w8 range m={m} n={n} k={k}", flush=True)
    rng = synth.stream(20, f"grad_w8/top/{m}x{k}")
    x = rng.standard_normal((m, k))
    x[rng.random((m, k)) < 2.0 / m] = 65504.0
    x[rng.random((m, k)) < 1.0 / m] = -64000.0
    x[m // 2, k // 2] = 65504.0
    x = torch.from_numpy(x.astype(np.float32)).half()
    dy = gradients(m, n, 21)
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    assert np.abs(xv).max() == 65536.0
    got = slim.grad_w8(dy.cuda(), slim.quant8(x.cuda()))
    check(got, dy.double().numpy(), xv)
    if k % 16 == 0:
        p, pick = kept(n, k)
        assert np.array_equal(host(slim.grad_w8(dy.cuda(), slim.quant8(x.cuda()), p)), pick(host(got)))


@pytest.mark.parametrize("m,n,k", SIZES)
@pytest.mark.parametrize("size", [2.0 ** 18, 1e12, 1e34])
def test_checkpoints_of_wider_types(m, n, k, size):
    # every third group holds rows of that size; the other groups' precision stays what it is
    print(f"grad_w8 range m={m} n={n} k={k} {size}", flush=True)
    rng = synth.stream(22, f"grad_w8/wide/{m}x{k}")
    x = rng.standard_normal((m, k))
    x *= np.where((np.arange(k) // 128 % 3 == 0) & (rng.random((m, 1)) < 0.3), size, 1.0)
    x[m // 2, 0] = size
    x = torch.from_numpy(x.astype(np.float32))
    dy = gradients(m, n, 23)
    xv = act8.values_rows(*act8.quant_rows(x.double().numpy()), k)
    check(slim.grad_w8(dy.cuda(), slim.quant8(x.cuda())), dy.double().numpy(), xv)


@pytest.mark.parametrize("m,n,k", [(700, 300, 500), (129, 2100, 4000)])
def test_groups_that_fit_are_untouched_by_one_that_does_not(m, n, k):
    rng = synth.stream(24, f"grad_w8/beside/{m}x{k}")
    x = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32))
    dy = gradients(m, n, 25).cuda()
    want = slim.grad_w8(dy, slim.quant8(x.cuda()))
    x[:, 128:256] *= 1e9
    got = slim.grad_w8(dy, slim.quant8(x.cuda()))
    assert torch.equal(got[:, :128], want[:, :128]) and torch.equal(got[:, 256:], want[:, 256:])


def test_nan_stays_in_its_column():
    x = torch.ones((600, 300))
    x[5, 7], x[6, 140] = 1e9, float("nan")
    g = slim.grad_w8(torch.ones((600, 130), device="cuda").half(), slim.quant8(x.cuda()))
    bad = g.isnan()
    assert bool(bad[:, 140].all()) and int(bad.sum()) == 130 and bool((g[:, 7] > 5e8).all())
