"""The router and the layer of experts against the oracle in 64 bits.

Bounds. Logits: fp32 products summed in chains of eight a lane, ten additions over lanes and waves and one for each 2048 columns, so
within L = (K / 256 + 80) 2^-24 (the sum of magnitudes) of their value; a weight is off by twice that relatively, and by 2^-20 for e^x and the
quotient. Experts: each product within 2^-17 of its magnitudes (at most 128 additions in a chain of the matrix unit's group and
fewer after it); an activation's slope below 1.13, its error below 2^-19 (|g| + 1); h is held to 2^-16; y is rounded by u |y|."""
import numpy as np
import pytest
import torch

from oracle import act8, mlp8
from paper_2608_24070_amd import slim
from tests.gpu_common import host, kernels_of

pytestmark = pytest.mark.gpu

DT = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
U = {"bf16": 2.0 ** -8, "fp16": 2.0 ** -11}
TINY = {"bf16": 2.0 ** -133, "fp16": 2.0 ** -24}


def gen(seed):
    return torch.Generator("cuda").manual_seed(seed)


def rows(m, k, dtype, g):
    """X as given to a call, and its values in 64 bits."""
    x = torch.randn((m, k), generator=g, device="cuda") * 2.0 ** torch.randint(-1, 2, (m, 1), generator=g, device="cuda")
    if dtype == "q8":
        q = slim.quant8(x.bfloat16())
        return q, act8.values_rows(host(q["codes"]), host(q["exps"]), k)
    x = x.to(DT[dtype])
    return x, host(x.double())


@pytest.mark.parametrize("m,e,k,top", [(1, 1, 1, 1), (1, 64, 4096, 8), (2, 5, 129, 5), (7, 8, 300, 2), (8, 512, 640, 16), (9, 65, 2051, 3),
                                       (61, 250, 8192, 6), (64, 64, 1000, 8), (300, 33, 512, 4)])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32", "q8"])
def test_route(m, e, k, top, dtype):
    for i, wt in enumerate(("fp32", "bf16", "fp16")):
        print(f"route m={m} e={e} k={k} top={top} {dtype} router {wt}", flush=True)
        g = gen(m + e + k + i)
        x, xv = rows(m, k, dtype, g)
        w = (torch.randn((e, k), generator=g, device="cuda") * k ** -0.5).to(DT[wt])
        wv = host(w.double())
        renorm = (m + i) % 2 == 0
        ids, p = slim.route(x, w, top, renorm=renorm)
        assert ids.dtype == torch.int32 and p.dtype == torch.float32 and ids.shape == p.shape == (m, top)
        ids, p = host(ids), host(p).astype(np.float64)
        logits, lim = xv @ wv.T, (k / 256 + 80) * 2.0 ** -24 * (np.abs(xv) @ np.abs(wv).T).max(1, keepdims=True)
        want, _ = mlp8.route(xv, wv, top, renorm)
        assert (ids >= 0).all() and (ids < e).all() and all(len(set(r)) == top for r in ids)
        # another order only where two logits are within their errors
        got_l, want_l = np.take_along_axis(logits, ids, 1), np.take_along_axis(logits, want, 1)
        assert (np.abs(got_l - want_l) <= 2 * lim).all()
        q = np.exp(logits - logits.max(1, keepdims=True))
        q /= q.sum(1, keepdims=True)
        r = np.take_along_axis(q, ids, 1)
        r = r / r.sum(1, keepdims=True) if renorm else r
        assert (np.abs(p - r) <= r * (4 * lim + 2.0 ** -19)).all()


def test_route_ties_go_to_the_lower_expert():
    x = torch.randn((5, 256), device="cuda").bfloat16()
    w = torch.randn((3, 256), device="cuda").bfloat16()
    many = w.repeat(100, 1)                     # expert e and e + 3, e + 6 .. alike
    ids, p = slim.route(x, many, 10)
    best = (x.float() @ w.float().t()).argmax(1, keepdim=True).int()
    assert torch.equal(ids, best + 3 * torch.arange(10, device="cuda", dtype=torch.int32))
    assert bool((p == p[:, :1]).all())
    ids, p = slim.route(torch.zeros_like(x), many, 4, renorm=False)
    assert ids.tolist() == [[0, 1, 2, 3]] * 5 and bool((p - 1 / 300).abs().max() < 1e-9)


def test_route_strides_and_far_logits():
    big = torch.randn((9, 700), device="cuda")
    x, w = big[1:7, 3:516], torch.randn((20, 600), device="cuda")[2:13, 5:518]
    ids, p = slim.route(x, w, 4)
    ids2, p2 = slim.route(x.contiguous(), w.contiguous(), 4)
    assert torch.equal(ids, ids2) and torch.equal(p, p2)
    # logits past what e^x holds, and an infinite one
    ids, p = slim.route(x * 1e4, w, 3, renorm=False)
    assert bool(p.isfinite().all()) and bool((p[:, 0] > 0.99).all())
    bad = x.clone()
    bad[2, 7] = float("nan")
    ids, p = slim.route(bad, w, 3)
    assert bool(p[2].isnan().all()) and bool(p[[0, 1, 3, 4, 5]].isfinite().all()) and bool((ids >= 0).all()) and bool((ids < 11).all())


def experts(e, d, f, g, gated=True):
    make = lambda n, k: torch.randn((e, n, k), generator=g, device="cuda") * k ** -0.5 * 2.0 ** torch.randint(-1, 2, (e, 1, 1), generator=g, device="cuda")
    ws = [make(f, d), make(f, d) if gated else None, make(d, f)]
    packs = [None if w is None else slim.pack8_experts(w) for w in ws]
    values = [None if w is None else [act8.values_weight(*act8.quant_weight(host(v).astype(np.float64))) for v in w] for w in ws]
    return packs, values


def check(Y, xv, values, ids, weights, act, res, dtype):
    gate, up, down = values
    ids, weights = host(ids), host(weights).astype(np.float64)
    m, d = xv.shape[0], down[0].shape[0]
    ref, lim = np.zeros((m, d)), np.zeros((m, d))
    for i in range(m):
        for e, w in zip(ids[i], weights[i]):
            if not 0 <= e < len(gate):
                continue
            x = xv[i]
            g, ge = gate[e] @ x, 2.0 ** -17 * (np.abs(gate[e]) @ np.abs(x))
            h, he = mlp8.value(act, g), 1.13 * ge + 2.0 ** -19 * (np.abs(g) + 1)
            if up is not None:
                u, ue = up[e] @ x, 2.0 ** -17 * (np.abs(up[e]) @ np.abs(x))
                h, he = h * u, he * (np.abs(u) + ue) + np.abs(h) * ue
            he = he + 2.0 ** -16 * np.abs(h)
            ref[i] += w * (down[e] @ h)
            lim[i] += abs(w) * (np.abs(down[e]) @ (he + 2.0 ** -17 * np.abs(h)) * (1 + 2.0 ** -10))
    if res is not None:
        ref = ref + host(res.double())
    got = host(Y.double())
    bad = ~(np.abs(got - ref) <= lim + U[dtype] * np.abs(ref) + TINY[dtype] + 2.0 ** -22 * np.abs(ref))
    assert not bad.any(), f"{bad.sum()} of {bad.size} out of bound, first {np.argwhere(bad)[:3].tolist()}"
    assert np.allclose(mlp8.experts(xv[:1], gate, up, down, ids[:1], weights[:1], act), ref[:1] - (0 if res is None else host(res.double())[:1]))


SIZES = [(1, 4, 128, 128, 2), (1, 16, 1000, 300, 8), (1, 3, 4096, 512, 1), (2, 9, 130, 17, 3), (7, 8, 512, 400, 2), (16, 5, 300, 129, 5),
         (33, 4, 260, 257, 2), (61, 40, 515, 170, 4), (64, 2, 384, 256, 1), (64, 3, 200, 1000, 3), (64, 100, 144, 130, 16), (20, 500, 128, 96, 8)]


@pytest.mark.parametrize("m,e,d,f,top", SIZES)
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "q8"])
def test_experts(m, e, d, f, top, dtype):
    i = m + e + d + f
    act, gated = list(mlp8.ACTS)[i % 5], i % 3 != 0
    out = "bf16" if dtype == "q8" else dtype
    print(f"moe8 m={m} e={e} d={d} f={f} top={top} {dtype} {act} gated={gated}", flush=True)
    g = gen(i)
    packs, values = experts(e, d, f, g, gated)
    x, xv = rows(m, d, dtype, g)
    ids, weights = slim.route(x, torch.randn((e, d), generator=g, device="cuda") * d ** -0.5, top)
    res = torch.randn((m, d), generator=g, device="cuda").to(DT[out]) if i % 2 else None
    Y = slim.moe8(x, *packs, ids, weights, act=act, residual=res)
    assert Y.shape == (m, d) and Y.dtype == DT[out]
    check(Y, xv, values, ids, weights, act, res, out)
    assert torch.equal(slim.moe8(x, *packs, ids, weights, act=act, residual=res), Y)
    # each row by itself gives the same to the bounds of both
    one = slim.moe8({"codes": x["codes"][:1], "exps": x["exps"][:1], "M": 1, "K": d} if dtype == "q8" else x[:1], *packs, ids[:1].contiguous(),
                    weights[:1].contiguous(), act=act, residual=None if res is None else res[:1])
    check(one, xv[:1], values, ids[:1], weights[:1], act, None if res is None else res[:1], out)


@pytest.mark.parametrize("m", [1, 5, 64])
def test_numbers_that_are_no_expert_and_ones_that_are_twice(m):
    g = gen(m)
    packs, values = experts(6, 300, 200, g)
    x, xv = rows(m, 300, "bf16", g)
    ids = torch.randint(-2, 9, (m, 5), generator=g, device="cuda", dtype=torch.int32)
    ids[0] = torch.tensor([3, -1, 3, 3, 6])
    weights = torch.rand((m, 5), generator=g, device="cuda")
    check(slim.moe8(x, *packs, ids, weights), xv, values, ids, weights, "silu", None, "bf16")
    # a row that is nowhere, alone and all of them: what it has on top of, and nothing else
    ids[m - 1] = torch.tensor([-1, 6, 99, -2147483648, 2147483647])
    res = torch.randn((m, 300), generator=g, device="cuda").bfloat16()
    assert torch.equal(slim.moe8(x, *packs, ids, weights, residual=res)[m - 1], res[m - 1])
    assert not bool(slim.moe8(x, *packs, torch.full_like(ids, -1), weights).any())
    # all rows at one expert
    ids.fill_(2)
    check(slim.moe8(x, *packs, ids, weights), xv, values, ids, weights, "silu", None, "bf16")


def test_nan_rows_stay_apart():
    g = gen(5)
    packs, _ = experts(4, 300, 200, g)
    x, _ = rows(30, 300, "bf16", g)
    ids = torch.randint(0, 4, (30, 2), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand((30, 2), generator=g, device="cuda")
    clean = slim.moe8(x, *packs, ids, weights)
    bad = x.clone()
    bad[3, 299], bad[20, 0] = float("nan"), float("inf")
    got = slim.moe8(bad, *packs, ids, weights)
    rest = torch.ones(30, dtype=torch.bool, device="cuda")
    rest[[3, 20]] = False
    assert bool(got[[3, 20]].isnan().any(1).all()) and torch.equal(got[rest], clean[rest])


def test_strides_places_and_the_bytes_around():
    g = gen(6)
    packs, _ = experts(4, 300, 200, g)
    wide = torch.randn((12, 400), generator=g, device="cuda").bfloat16()
    x = wide[1:10, 7:307]
    ids = torch.randint(0, 4, (9, 2), generator=g, device="cuda", dtype=torch.int32)
    weights = torch.rand((9, 2), generator=g, device="cuda")
    want = slim.moe8(x.contiguous(), *packs, ids, weights, residual=x.contiguous())
    # NaN around the rows is not read
    wide[0], wide[10:], wide[:, :7], wide[:, 307:] = (float("nan"),) * 4
    buf = torch.full((11, 333), -7.0, dtype=torch.bfloat16, device="cuda")
    out = buf[1:10, 5:305]
    slim.moe8(x, *packs, ids, weights, residual=x, out=out)
    assert torch.equal(out, want)
    out.copy_(x)
    assert torch.equal(slim.moe8(x, *packs, ids, weights, residual=out, out=out), want)
    # in the rows' own place
    out.copy_(x)
    assert torch.equal(slim.moe8(out, *packs, ids, weights, residual=out, out=out), want)
    out.fill_(-7.0)
    assert bool((buf == -7).all())


@pytest.mark.parametrize("m,e,d,f,top", [(1, 16, 512, 256, 4), (61, 10, 515, 170, 4)])
def test_streams_graph_replays_and_workspaces(m, e, d, f, top):
    g = gen(9)
    packs, _ = experts(e, d, f, g)
    x, _ = rows(m, d, "bf16", g)
    router = torch.randn((e, d), generator=g, device="cuda") * d ** -0.5

    def call(stream=None):
        ids, weights = slim.route(x, router, top, stream=stream)
        return slim.moe8(x, *packs, ids, weights, residual=x, stream=stream), ids, weights

    same = lambda a, b: all(torch.equal(s, t) for s, t in zip(a, b))
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = call(side)
    side.synchronize()
    assert same(got, want)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = call()
    for rep in range(3):
        x.normal_()
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert same(held, call()), rep
    # exactly the workspace that is asked for
    ids, weights = slim.route(x, router, top)
    for need, run in ((slim.slim_moe8_workspace(m, d, f, e, top), lambda ws: slim.moe8(x, *packs, ids, weights, ws=ws)),
                      (slim.slim_route_workspace(m, e, d), lambda ws: slim.route(x, router, top, ws=ws)[1])):
        ws = torch.full((need + 256,), 0xFF, dtype=torch.uint8, device="cuda")
        got = run(ws[:need])
        assert bool((ws[need:] == 0xFF).all()) and torch.equal(got, run(None))
        with pytest.raises(slim.SlimError):
            run(ws[:need - 1])


def test_two_streams_at_once():
    g = gen(13)
    packs, _ = experts(8, 512, 640, g)
    router = torch.randn((8, 512), generator=g, device="cuda") * 512 ** -0.5
    w1 = slim.pack8(torch.randn((1024, 512), generator=g, device="cuda") / 22)
    xs = [rows(m, 512, "bf16", g)[0] for m in (48, 61)]

    def work(x):
        ids, weights = slim.route(x, router, 3)
        y = slim.moe8(x, *packs, ids, weights, residual=x)
        q = slim.linear8_act(y, w1, act="gelu", q8=True)
        return [ids, weights, y, q["codes"], q["exps"]]

    want = [work(x) for x in xs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in xs]
    got = []
    for _ in range(20):
        for x, s in zip(xs, streams):
            with torch.cuda.stream(s):
                got.append(work(x))
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for i, r in enumerate(got) for a, b in zip(r, want[i % 2]))


def test_no_rows():
    g = gen(1)
    packs, _ = experts(3, 128, 128, g)
    x = torch.empty((0, 128), dtype=torch.bfloat16, device="cuda")
    ids, weights = slim.route(x, torch.zeros((3, 128), device="cuda"), 2)
    assert ids.shape == (0, 2) and slim.moe8(x, *packs, ids, weights).shape == (0, 128)


def test_a_block_of_layers_together():
    """The 8-bit path's MLP with its new pieces, as a transformer block has them: norm, router, experts and residual; norm, gated
    product and the product that adds to the block's input."""
    g = gen(11)
    d, f, e, m = 512, 640, 8, 24
    packs, values = experts(e, d, f, g)
    x = torch.randn((m, d), generator=g, device="cuda").bfloat16()
    n, _, _ = slim.norm(x, rms=True, q8=True)
    router = torch.randn((e, d), generator=g, device="cuda") * d ** -0.5
    ids, weights = slim.route(n, router, 2)
    y = slim.moe8(n, *packs, ids, weights, residual=x)
    check(y, act8.values_rows(host(n["codes"]), host(n["exps"]), d), values, ids, weights, "silu", x, "bf16")
    w = [torch.randn(s, generator=g, device="cuda") * s[1] ** -0.5 for s in ((f, d), (f, d), (d, f))]
    pg, pu, pd = (slim.pack8(v) for v in w)
    n2, _, _ = slim.norm(y, rms=True, q8=True)
    h = slim.linear8_act(n2, pg, act="silu", mul=slim.linear8(n2, pu), q8=True)
    z = slim.linear8_act(h, pd, residual=y)
    nv = slim.dequant8(n2, torch.float32).double()
    wide = [torch.from_numpy(act8.values_weight(*act8.quant_weight(host(v).astype(np.float64)))).cuda() for v in w]
    hv = torch.nn.functional.silu(nv @ wide[0].t()) * (nv @ wide[1].t())
    ref = hv @ wide[2].t() + y.double()
    # h's rounding to 8 bits (2^-4 at most, uniform: a third of it on average) over its own sum of 640, up's to 16
    err = 2.0 ** -4 * (hv.abs() @ wide[2].t().abs()) + 2.0 ** -8 * ref.abs()
    assert bool(((z.double() - ref).abs() <= err).all()) and bool(((z.double() - ref).norm() / ref.norm()) < 2.0 ** -4)


def test_the_kernels_that_run():
    g = gen(2)
    packs, _ = experts(4, 512, 256, g)
    x, _ = rows(3, 512, "bf16", g)
    router = torch.randn((4, 512), generator=g, device="cuda")
    ids, weights = slim.route(x, router, 2)
    assert kernels_of(lambda: slim.route(x, router, 2)) == {"route_logits", "route_top"}
    assert {"moe_up", "moe_down"} <= kernels_of(lambda: slim.moe8(x, *packs, ids, weights))
