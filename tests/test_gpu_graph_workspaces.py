"""Graphs of calls that were given no workspace, replayed after larger calls on the stream of their capture: right results, and
no write to memory that others hold by then."""
import pytest
import torch

from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu


def replays_keep_to_their_own(small, large, outs):
    """small() is warmed up and captured on one stream, large() follows there; then the allocator gives out what it has, and
    every replay has to leave that as it is and to give small()'s results (`outs`: its tensors, from the captured call's)."""
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        want = [t.clone() for t in outs(small())]
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = outs(small())
    with torch.cuda.stream(side):
        large()
        others = [torch.full((n,), 7, dtype=torch.uint8, device="cuda") for n in (1 << 16, 1 << 18, 1 << 20, 1 << 22) for _ in range(8)]
    side.synchronize()
    for i in range(3):
        for t in got:
            t.fill_(3.0)
        torch.cuda.synchronize()
        graph.replay()
        with torch.cuda.stream(side):
            large()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
        assert all(bool((t == 7).all()) for t in others), i


def rows(m, k, seed=0):
    return torch.randn((m, k), generator=torch.Generator("cuda").manual_seed(seed), device="cuda").bfloat16()


def test_linear8():
    p = slim.pack8(rows(512, 2048).float())
    a, b = rows(24, 2048, 1), rows(3000, 2048, 2)
    replays_keep_to_their_own(lambda: slim.linear8(a, p), lambda: slim.linear8(b, p), lambda y: [y])


def test_grad_w8():
    qa, qb = slim.quant8(rows(2600, 256)), slim.quant8(rows(9000, 256, 1))
    da, db = rows(2600, 130, 2), rows(9000, 130, 3)
    replays_keep_to_their_own(lambda: slim.grad_w8(da, qa), lambda: slim.grad_w8(db, qb), lambda y: [y])


def test_norm_bwd():
    a, b = rows(300, 1000), rows(5000, 8192, 1)
    sa, sb = slim.norm(a)[1:], slim.norm(b)[1:]
    replays_keep_to_their_own(lambda: slim.norm_bwd(a, a, None, *sa), lambda: slim.norm_bwd(b, b, None, *sb), list)
