"""Experts of one and two rows whose down product is in parts of the reduction: eight waves on 16 columns, a wave's groups within or across
the row's picks, fp32 sums in memory and a launch that adds them. Bounds as in test_gpu_moe8."""
import pytest
import torch

from oracle import mlp8
from paper_2608_24070_amd import slim
from tests.gpu_common import kernels_of
from tests.test_gpu_moe8 import DT, check, experts, gen, rows

pytestmark = pytest.mark.gpu

# parts: 2, 2, 4, 2, 16 (the most), 2
SIZES = [(1, 8, 300, 2100, 8), (2, 8, 300, 2100, 8), (1, 9, 512, 4096, 8), (1, 3, 256, 11008, 2), (1, 2, 100, 70000, 2), (2, 5, 384, 4097, 4)]


def parts(m, d, f, e, top):
    """How many sums of the results the workspace holds behind h (two 16-bit values for each pair and group's column)."""
    h = -(-(m * top * -(-f // 128) * 128 * 2) // 256) * 256
    table = 0 if m == 1 else 16 + 512 * 16 + 2 * 4 * 64 * 16          # experts and their places, a row and a weight each
    left = slim.slim_moe8_workspace(m, d, f, e, top) - 2 * h - -(-table // 256) * 256
    return left // (m * d * 4)


@pytest.mark.parametrize("m,e,d,f,top", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "q8"])
def test_parts_of_one_and_two_rows(m, e, d, f, top, dtype):
    i = m + e + d + f
    act, out = list(mlp8.ACTS)[i % 5], "bf16" if dtype == "q8" else dtype
    assert parts(m, d, f, e, top) > 1
    print(f"moe8 in parts m={m} e={e} d={d} f={f} top={top} {dtype} {act}", flush=True)
    g = gen(i)
    packs, values = experts(e, d, f, g, i % 3 != 0)
    x, xv = rows(m, d, dtype, g)
    ids, weights = slim.route(x, torch.randn((e, d), generator=g, device="cuda") * d ** -0.5, top)
    res = torch.randn((m, d), generator=g, device="cuda").to(DT[out])
    call = lambda **kw: slim.moe8(x, *packs, ids, weights, act=act, **kw)
    ran = kernels_of(lambda: call(residual=res))
    assert ran == {"moe_up", "moe_down", "moe_sum"} | ({"moe_table"} if m > 1 else set())
    Y = call(residual=res)
    check(Y, xv, values, ids, weights, act, res, out)
    check(call(), xv, values, ids, weights, act, None, out)
    assert torch.equal(call(residual=res), Y)
    # in the residual's place, columns of a wider buffer
    wide = torch.full((m, d + 9), -7.0, dtype=DT[out], device="cuda")
    wide[:, 3:3 + d] = res
    assert torch.equal(call(residual=wide[:, 3:3 + d], out=wide[:, 3:3 + d]), Y)
    wide[:, 3:3 + d] = -7.0
    assert bool((wide == -7).all())


@pytest.mark.parametrize("m", [1, 2])
def test_numbers_twice_and_of_no_expert(m):
    e, d, f, top = 6, 300, 4100, 8
    assert parts(m, d, f, e, top) > 1
    g = gen(m)
    packs, values = experts(e, d, f, g)
    x, xv = rows(m, d, "bf16", g)
    weights = torch.rand((m, top), generator=g, device="cuda")
    for picks in ([3, -1, 3, 3, 6, 0, 5, 0], [-1, 6, 99, -2147483648, 2147483647, 4, -7, 4], [2] * 8, [0, 1, 2, 3, 4, 5, 0, 1], [-1] * 7 + [5]):
        ids = torch.tensor([picks] * m, dtype=torch.int32, device="cuda")
        ids[m - 1] = ids[m - 1].flip(0)
        check(slim.moe8(x, *packs, ids, weights), xv, values, ids, weights, "silu", None, "bf16")
    res = torch.randn((m, d), generator=g, device="cuda").bfloat16()
    assert torch.equal(slim.moe8(x, *packs, torch.full_like(ids, 6), weights, residual=res), res)


def test_a_graph_of_parts():
    m, e, d, f, top = 1, 8, 300, 2100, 8
    g = gen(3)
    packs, _ = experts(e, d, f, g)
    x, _ = rows(m, d, "bf16", g)
    router = torch.randn((e, d), generator=g, device="cuda")

    def call():
        ids, weights = slim.route(x, router, top)
        return slim.moe8(x, *packs, ids, weights, residual=x)

    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for _ in range(3):
        x.normal_()
        held.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held, call())
