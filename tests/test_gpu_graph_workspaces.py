"""Graphs of calls that were given no workspace, replayed after larger calls on the stream of their capture: right results, and
no write to memory that others hold by then."""
import numpy as np
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


# ------------------------------------------------------------------ the compressed layer
def layer(n, k, r, seed=0):
    g = torch.Generator("cuda").manual_seed(seed)
    half = lambda *s: torch.randn(s, generator=g, device="cuda").half()
    p = slim.pack(torch.randn((n, k), generator=g, device="cuda"))
    return p, slim.pack_adapter(half(k, r) * k ** -0.5, half(r, n)), slim.pack_bwd(p), half(k, r) * k ** -0.5, half(r, n)


@pytest.mark.parametrize("m", [4, 16, 100, 700])
def test_linear(m):
    p, ad, pb, L, R = layer(1024, 2048, 64)
    a, b = rows(m, 2048), rows(5000, 2048, 1)
    replays_keep_to_their_own(lambda: slim.linear(a, p, ad), lambda: slim.linear(b, p, ad), lambda y: [y])


@pytest.mark.parametrize("m", [16, 300])
def test_bwd_dx(m):
    p, ad, pb, L, R = layer(1024, 1024, 64)
    a, b = rows(m, 1024), rows(5000, 1024, 1)
    replays_keep_to_their_own(lambda: slim.bwd_dx(a, pb, L, R), lambda: slim.bwd_dx(b, pb, L, R), lambda y: [y])


@pytest.mark.parametrize("m", [16, 300])
def test_linear_qa(m):
    p, ad, pb, L, R = layer(1024, 2048, 64)
    q = slim.pack_adapter_q(L, R)
    a, b = rows(m, 2048), rows(5000, 2048, 1)
    replays_keep_to_their_own(lambda: slim.linear_qa(a, p, q), lambda: slim.linear_qa(b, p, q), lambda y: [y])


def test_a_graph_does_not_need_another_ones_replay():
    # no call before the captures on their stream, and the second graph runs first: its control words are its own to clear
    p, ad, *_ = layer(4096, 4096, 384)
    a, b = rows(16, 4096), rows(7, 4096, 1)
    want = slim.linear(a, p, ad), slim.linear(b, p, ad)
    torch.cuda.synchronize()
    side, graphs, got = torch.cuda.Stream(), [], []
    for x in (a, b):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=side):
            got.append(slim.linear(x, p, ad))
    for i in (1, 0, 1, 1, 0, 0):
        got[i].fill_(3.0)
        graphs[i].replay()
        torch.cuda.synchronize()
        assert torch.equal(got[i], want[i]), i
        with torch.cuda.stream(side):
            assert torch.equal(slim.linear(b, p, ad), want[1])
        side.synchronize()


def test_a_given_stream_clears_its_workspace():
    # the fill and the layer are on the given stream, so that the layer finds its control words clear
    p, ad, *_ = layer(1024, 2048, 64)
    a = rows(8, 2048)
    want = slim.linear(a, p, ad)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    got = slim.linear(a, p, ad, stream=s)
    s.synchronize()
    assert torch.equal(got, want) and slim.workspace(1, a.device, s).is_cuda
    assert s.cuda_stream in {stream for dev, stream in slim._ws_cache}


def test_linear_hybrid():
    # a reduction in splits, whose partials are in the workspace
    kinds = np.ones((4, 32), dtype=np.uint8)
    p = slim.pack_hybrid(torch.randn((512, 4096), generator=torch.Generator("cuda").manual_seed(0), device="cuda"), kinds)
    a, b = rows(128, 4096).half(), rows(2048, 4096, 1).half()
    assert 0 < slim.slim_linear_hybrid_workspace(128, 512, 4096) < slim.slim_linear_hybrid_workspace(2048, 512, 4096)
    replays_keep_to_their_own(lambda: slim.linear_hybrid(a, p), lambda: slim.linear_hybrid(b, p), lambda y: [y])
