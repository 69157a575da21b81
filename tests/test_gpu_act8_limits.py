"""The ends of the 8-bit format's range, against the values of its definition rounded to each type by torch on the host."""
import numpy as np
import pytest
import torch

from oracle import act8
from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu


def both(x, dtype):
    """dequant8(quant8(x)) in dtype, and the definition's values rounded to it."""
    t = torch.tensor([x], dtype=torch.float32)
    want = torch.from_numpy(act8.values_rows(*act8.quant_rows(t.double().numpy()), len(x)))
    return slim.dequant8(slim.quant8(t.cuda()), dtype).cpu(), want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_largest_values(dtype):
    # at e = 120: 247 2^120 is nearest to 240 2^120, from 248 2^120 on 256 2^120 = 2^128 is, which the types do not hold
    top = torch.finfo(torch.float32).max
    got, want = both([247 * 2.0 ** 120, -247 * 2.0 ** 120, 248 * 2.0 ** 120, top, -top, 1.0], dtype)
    assert want[0].tolist() == [240 * 2.0 ** 120, -240 * 2.0 ** 120, 2.0 ** 128, 2.0 ** 128, -2.0 ** 128, 0.0]
    assert got[0].tolist() == [240 * 2.0 ** 120, -240 * 2.0 ** 120, np.inf, np.inf, -np.inf, 0.0]


def test_smallest_values():
    # e = -126: multiples of 2^-135, exact in fp32; bf16 has multiples of 2^-133, exact from 2^-130 on
    x = [2.0 ** -135 * i for i in range(-20, 300)]
    got, want = both(x, torch.float32)
    assert torch.equal(got.double(), want)
    big = want.abs() >= 2.0 ** -130
    got = both(x, torch.bfloat16)[0].double()
    assert torch.equal(got[big], want[big])
    assert bool(((got - want).abs() <= 2.0 ** -134).all())
