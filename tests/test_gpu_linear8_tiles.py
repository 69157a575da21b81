"""slim_linear8 at sizes for which each of its tile kernels is picked: last tiles of a few rows or columns, reductions that end
inside a part, one group or many.

Integers of -2 .. 2 in a fifth of the places make every sum a small integer that fp16 holds, so the whole result is compared
exactly; values of other sizes are compared at some rows, with the bound of the product's other tests."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim, synth
from tests.gpu_common import host
from tests.test_gpu_linear8 import check

pytestmark = pytest.mark.gpu

# by tile: 64 x 64, 64 x 128, 128 x 128, 128 x 256, 192 x 256, 256 x 256
SIZES = [(65, 17, 129), (100, 513, 1300), (200, 130, 4100),
         (129, 1000, 129), (2047, 100, 900), (300, 2050, 2100),
         (1500, 2050, 1300), (700, 5000, 2100),
         (400, 8200, 129), (2047, 2050, 300), (8192, 513, 640),
         (1000, 8200, 129), (2500, 4100, 900), (4097, 2050, 1300),
         (1500, 8200, 129), (2500, 5000, 640), (6001, 2050, 1100)]
# few tiles and a long reduction, which is then sliced: of each tile kernel that can be, with slices that end past the last group
SLICED = [(5, 130, 28672), (24, 512, 14336), (64, 1000, 28001), (100, 513, 28672), (300, 131, 9000), (512, 515, 28672), (1024, 770, 20001),
          (2000, 200, 12345)]


@pytest.mark.parametrize("m,n,k", SIZES + SLICED)
def test_small_integers_are_exact(m, n, k):
    print(f"linear8 tiles m={m} n={n} k={k}", flush=True)
    gen = torch.Generator("cuda").manual_seed(m + n + k)
    ints = lambda r: torch.randint(-2, 3, (r, k), generator=gen, device="cuda") * (torch.rand((r, k), generator=gen, device="cuda") < 0.2)
    x, w = ints(m).float(), ints(n).float()
    buf = torch.full((m + 1, n + 8), 9.0, dtype=torch.float16, device="cuda")
    slim.linear8(slim.quant8(x), slim.pack8(w), out=buf[:m, :n])
    assert torch.equal(buf[:m, :n].float(), x @ w.T)
    assert bool((buf[m] == 9).all()) and bool((buf[:, n:] == 9).all())


@pytest.mark.parametrize("m,n,k", SIZES + SLICED)
@pytest.mark.parametrize("out", [torch.bfloat16, torch.float16])
def test_values_of_any_size(m, n, k, out):
    print(f"linear8 tiles m={m} n={n} k={k} {out}", flush=True)
    gen = torch.Generator("cuda").manual_seed(m + n + k + 1)
    spread = lambda r: 4.0 ** torch.randint(-2, 3, (r, 1), generator=gen, device="cuda")
    x = torch.randn((m, k), generator=gen, device="cuda") * spread(m)
    w = torch.randn((n, k), generator=gen, device="cuda") * spread(n) / 50
    Y = slim.linear8(x, slim.pack8(w), dtype=out)
    rows = np.unique(np.r_[0, m - 1, synth.stream(0, f"linear8/rows/{m}").integers(0, m, 40)])
    xv = act8.values_rows(*act8.quant_rows(host(x)[rows].astype(np.float64)), k)
    wv = act8.values_weight(*act8.quant_weight(host(w).astype(np.float64)))
    check(Y[torch.from_numpy(rows).cuda()], xv, wv, "bf16" if out is torch.bfloat16 else "fp16")


@pytest.mark.parametrize("m,n,k", SLICED)
def test_slices_are_what_runs(m, n, k):
    x, p = torch.zeros((m, k), dtype=torch.bfloat16, device="cuda"), slim.pack8(torch.zeros((n, k), device="cuda"))
    slim.slim_timing_reset()
    slim.slim_timing_enable(True)
    Y = slim.linear8(x, p)
    torch.cuda.synchronize()
    slim.slim_timing_enable(False)
    assert {"linear8_tile", "linear8_sum"} <= set(slim.slim_timing_read()) and not bool(Y.any())
    # the workspace is exactly what is asked for: nothing is written past it
    q = slim.quant8(x)
    need = slim.slim_linear8_workspace(slim.SLIM_Q8_E4M3, m, n, k)
    ws = torch.full((need + 256,), 7, dtype=torch.uint8, device="cuda")
    slim.linear8(q, p, ws=ws[:need])
    assert need > 0 and bool((ws[need:] == 7).all())
    with pytest.raises(slim.SlimError):
        slim.linear8(q, p, ws=ws[:need - 16])
