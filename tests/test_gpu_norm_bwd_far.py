"""slim_norm_bwd for rows whose mean times rstd passes fp32's range while every deviation is small: what lies past a row's end
takes no part. Rows of one value 2^120, with the statistics of such rows: xh = 0, so dgamma = 0 and dx = rstd (t - mean t).

Bound: dx in u of itself (u the last half place of its type) and 64 2^-24 of its two terms; the sums of a row add K values of
either sign in chains of at most 8 V + 16 (V <= 8 vectors a thread), fewer than 64."""
import numpy as np
import pytest
import torch

from paper_2608_24070_amd import slim, synth
from tests.gpu_common import host

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp32": 2.0 ** -24}
VALUE = 2.0 ** 120


@pytest.mark.parametrize("k", [1, 9, 100, 512, 520, 1000, 1021, 2000, 4097, 5120, 8191, 9000, 12289, 16384, 20000, 28671, 28680])
@pytest.mark.parametrize("dtype,q8", [("bf16", False), ("fp32", False), ("bf16", True), ("fp32", True)])
def test_rows_of_one_huge_value(k, dtype, q8):
    print(f"norm_bwd far k={k} {dtype} q8={q8}", flush=True)
    m = 5
    rng = synth.stream(30, f"norm/huge/{k}")
    x = torch.full((m, k), VALUE, dtype=DT[dtype], device="cuda")
    dy = torch.from_numpy(rng.standard_normal((m, k)).astype(np.float32)).to(DT[dtype])
    g = torch.from_numpy((1 + 0.3 * rng.standard_normal(k)).astype(np.float32))
    mean = torch.full((m,), VALUE, device="cuda")
    rstd = torch.full((m,), 316.0, device="cuda")
    dx, dg, db = slim.norm_bwd(dy.cuda(), slim.quant8(x) if q8 else x, g.cuda(), mean, rstd)
    t = dy.double().numpy() * g.double().numpy()
    tm = t.mean(1, keepdims=True)
    ref = 316.0 * (t - tm)
    lim = U[dtype] * np.abs(ref) + 64 * 2.0 ** -24 * 316.0 * (np.abs(t) + np.abs(t).mean(1, keepdims=True))
    got = dx.double().cpu().numpy()
    assert np.all(np.isfinite(got)) and np.all(np.abs(got - ref) <= lim)
    assert bool((dg == 0).all())
    assert np.all(np.abs(host(db) - dy.double().numpy().sum(0)) <= (m + 64) * 2.0 ** -24 * np.abs(dy.double().numpy()).sum(0))
