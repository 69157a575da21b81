"""Every path that a product with an activation at its end can take is one that the GPU tests' sizes take: the library's own plan, over
random sizes, against that of those sizes."""
import random

import pytest

from tests import test_gpu_linear8_act as t, test_gpu_linear8_act_paths as more
from tests.plans import act_plan

# direction, 8-bit results (the backward's groups)
CALLS = [(False, False), (False, True), (True, True)]


def path(bwd, groups, m, n, k):
    p = act_plan(bwd, m, n, k, groups)
    assert p.few or (0 <= p.kind < 6 and p.slices >= 1)
    return (("few", p.few) if p.few else ("tile", p.kind)), p.direct, p.slices > 1


@pytest.mark.parametrize("bwd,groups", CALLS)
def test_the_sizes_take_every_path(bwd, groups):
    took = {path(bwd, groups, *s) for s in t.FEW + t.TILES + t.SLICED + more.SIZES}
    rng = random.Random(8)
    size = lambda lo, hi: int(lo * (hi / lo) ** rng.random())
    for _ in range(30000):
        s = size(1, 9000), size(1, 30000), size(1, 30000)
        assert path(bwd, groups, *s) in took, s
    tile = lambda kind, direct, sliced: (("tile", kind), direct, sliced) in took
    assert all(tile(k, True, False) for k in range(5)) and all(tile(k, False, True) for k in (3, 4, 5)) and tile(5, False, False)
    assert all(((("few", f), not (bwd or groups), False) in took) for f in (1, 2, 4))


@pytest.mark.parametrize("bwd,groups", CALLS)
def test_the_paths_of_the_sizes(bwd, groups):
    # what the sizes of the file of their own are there for
    want = [("tile", 3), ("tile", 3), ("tile", 5), ("tile", 5)]
    for s, kernel in zip(more.SIZES, want):
        p = act_plan(bwd, *s, groups)
        assert (("few", p.few) if p.few else ("tile", p.kind)) == kernel and not p.direct and (p.slices > 1) == (kernel == ("tile", 3)), s
