"""Activations and weights in 8 bits (slim_quant8, slim_dequant8, slim_pack8) against the oracle: equal to the bit."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim, synth
from tests.gpu_common import dev, host

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


def rows(m, k, dtype, seed=0, name="act8"):
    """A device tensor with rows of very different sizes, zeros, a zero row, and its float64 values."""
    rng = synth.stream(seed, f"{name}/{m}x{k}/{dtype}")
    lo, hi = (-6, 4) if dtype == "fp16" else (-30, 30)
    x = rng.standard_normal((m, k)) * 10.0 ** rng.uniform(lo, hi, (m, 1))
    x *= np.where(rng.random((m, k)) < 0.05, 0.0, 1.0) * np.where(rng.random((m, k)) < 0.02, 30.0, 1.0)
    if m > 2:
        x[m // 2] = 0.0
    x = np.clip(x, -60000, 60000) if dtype == "fp16" else x
    t = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
    return t.cuda(), t.double().numpy()


def same_rows(q, x):
    codes, exps = act8.quant_rows(x)
    assert np.array_equal(host(q["exps"]), exps)
    assert np.array_equal(host(q["codes"]), codes)


@pytest.mark.parametrize("m,k", [(1, 1), (1, 4096), (3, 127), (5, 128), (7, 129), (33, 511), (9, 513), (300, 4097), (2, 28672)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_quant_and_back(m, k, dtype):
    print(f"quant8 m={m} k={k} {dtype}", flush=True)
    t, x = rows(m, k, dtype)
    q = slim.quant8(t)
    same_rows(q, x)
    v = act8.values_rows(host(q["codes"]), host(q["exps"]), k)
    for out in ("fp32", "bf16", dtype):
        got = slim.dequant8(q, DT[out])
        want = torch.from_numpy(v.astype(np.float32)).to(DT[out])     # exact in fp32; one rounding to 16 bits
        assert torch.equal(got.cpu(), want), out


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_every_rounding_case(dtype):
    # all codes and the points around their midpoints, with the group's largest value at 448 or just past it
    v = act8.VALUES[:127]
    mid = (v[1:] + v[:-1]) / 2
    pts = np.concatenate([v, mid, mid * (1 + 2.0 ** -7), mid * (1 - 2.0 ** -7)])
    pts = np.concatenate([pts, -pts])
    for top in (448.0, 450.0, 447.0):
        x = np.zeros((len(pts) // 64 + 1, 128))
        flat = np.concatenate([pts, np.zeros((-len(pts)) % 64)]).reshape(-1, 64)
        x[: len(flat), 1:65] = flat
        x[:, 0] = top
        t = torch.from_numpy(x.astype(np.float32)).to(DT[dtype])
        same_rows(slim.quant8(t.cuda()), t.double().numpy())


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_nan_and_infinity_stay_their_own(dtype):
    t, x = rows(6, 300, dtype, seed=3)
    x = x.copy()
    for r, c, v in ((0, 5, np.nan), (1, 130, np.inf), (2, 299, -np.inf), (2, 0, np.nan)):
        x[r, c] = v
        t[r, c] = float(v)
    q = slim.quant8(t)
    codes, exps = act8.quant_rows(x)
    assert np.array_equal(host(q["exps"]), exps)
    # a NaN's sign is of no account
    got = host(q["codes"])
    assert np.array_equal(np.where(got == 0xFF, 0x7F, got), np.where(codes == 0xFF, 0x7F, codes))
    back = host(slim.dequant8(q, torch.float32))
    assert np.array_equal(np.isnan(back), ~np.isfinite(x))


def test_smallest_values_of_fp32_keep_the_least_exponent():
    x = np.full((2, 128), 2.0 ** -140)
    x[1, 3] = 2.0 ** -126
    same_rows(slim.quant8(dev(x.astype(np.float32))), x)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_rows_of_any_stride_and_start(dtype):
    t, _ = rows(40, 1000, dtype, seed=4)
    view = t[3:20, 7:7 + 393]
    q = slim.quant8(view)
    same_rows(q, view.double().cpu().numpy())
    out = torch.full((17, 500), -7.0, dtype=DT[dtype], device="cuda")
    slim.dequant8(q, out=out[:, 5:5 + 393])
    assert torch.equal(out[:, 5:398], slim.dequant8(q, DT[dtype]))
    assert bool((out[:, :5] == -7).all()) and bool((out[:, 398:] == -7).all())


def test_no_rows():
    q = slim.quant8(torch.empty((0, 200), dtype=torch.bfloat16, device="cuda"))
    assert q["codes"].shape == (0, 256) and slim.dequant8(q).shape == (0, 200)


@pytest.mark.parametrize("n,k", [(1, 1), (16, 128), (17, 129), (128, 128), (200, 300), (513, 640)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_pack8_both_ways(n, k, dtype):
    print(f"pack8 n={n} k={k} {dtype}", flush=True)
    t, x = rows(n, k, dtype, seed=5)
    p = slim.pack8(t, bwd=True)
    codes, e = act8.quant_weight(x)
    assert np.array_equal(host(p["codes"]), act8.tiles(codes)) and np.array_equal(host(p["exps"]), act8.exponent_rows(e))
    assert np.array_equal(host(p["codesT"]), act8.tiles(codes.T)) and np.array_equal(host(p["expsT"]), act8.exponent_rows(e.T))
    f = slim.pack8(t)
    assert "codesT" not in f and torch.equal(f["codes"], p["codes"])


def test_pack8_of_a_view():
    t, _ = rows(200, 400, "bf16", seed=6)
    view = t[9:150, 3:260]
    codes, e = act8.quant_weight(view.double().cpu().numpy())
    p = slim.pack8(view)
    assert np.array_equal(host(p["codes"]), act8.tiles(codes)) and np.array_equal(host(p["exps"]), act8.exponent_rows(e))
