"""The example that trains and serves one MLP block on the 8-bit path, against the block in 64 bits.

Rounding to e4m3 moves a value by at most half a step, and a step is 2^-3 of the power of two below the value: as a random
error at most 2^-3 / sqrt(12) = 0.036 of it. On the way to any of the results lie at most ten such roundings (three
operands and their weights forward, three backward, the kept input), independent of one another: sqrt(10) 0.036 = 0.114 of
the result's norm."""
import pytest
import torch
import torch.nn.functional as F

from examples.mlp8 import MLP8, kept_bytes, train

pytestmark = pytest.mark.gpu

ROUNDED = 0.114


def rel(got, want):
    return float((got.double().cpu() - want).norm() / want.norm())


def block(x, model, rms):
    """The block and its parameters as 64-bit leaves on the CPU."""
    leaf = lambda t: t.double().cpu().requires_grad_()
    p = {"w1": leaf(model.w1), "w2": leaf(model.w2), "gamma": leaf(model.gamma)}
    if not rms:
        p["beta"] = leaf(model.beta)
    mu = 0 if rms else x.mean(1, keepdim=True)
    n = (x - mu) * ((x - mu).square().mean(1, keepdim=True) + 1e-5).rsqrt() * p["gamma"] + (0 if rms else p["beta"])
    return x + F.gelu(n @ p["w1"].T) @ p["w2"].T, p


@pytest.mark.parametrize("tokens,d,ffn", [(1, 128, 256), (33, 256, 384), (500, 512, 1408)])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("sparse", [False, True])
def test_against_64_bits(tokens, d, ffn, rms, sparse):
    model = MLP8(d, ffn, sparse, rms, seed=3)
    g = torch.Generator("cuda").manual_seed(4)
    x, dy = (torch.randn((tokens, d), generator=g, device="cuda").bfloat16() for _ in range(2))
    y, kept = model.forward(x)
    dx, grads = model.backward(dy, kept)
    x64 = x.double().cpu().requires_grad_()
    want, p = block(x64, model, rms)
    want.backward(dy.double().cpu())
    assert rel(y, want.detach()) < ROUNDED and rel(dx, x64.grad) < ROUNDED
    for name, leaf in p.items():
        ref = leaf.grad
        if sparse and name == "w2":
            ref = ref[model.kept.cpu()].view(d, ffn // 2)
        assert rel(grads[name], ref) < ROUNDED, name
    assert rms == (grads["beta"] is None)
    # a byte a value, an exponent a group in whole words, and the norm's statistics
    words = lambda k: -(-k // 512) * 4
    assert kept_bytes(kept) == tokens * (2 * (d + words(d)) + 2 * (ffn + words(ffn)) + 4 * (1 if rms else 2))


@pytest.mark.parametrize("sparse", [False, True])
def test_training_lowers_the_error_and_keeps_the_pattern(sparse):
    model = MLP8(256, 512, sparse)
    losses = train(model, 512, 60, lr=0.01, decay=0.01)
    assert sum(losses[-5:]) < 0.8 * sum(losses[:5]), losses
    if sparse:
        assert bool((model.w2[~model.kept] == 0).all()) and bool((model.kept.view(256, -1, 4).sum(2) == 2).all())
        assert torch.equal(model.values["vals"].view(torch.float16).float().flatten(), model.w2[model.kept].half().float())


def test_single_tokens_are_rows_of_the_batch():
    # other kernels sum in another order; a half place of bf16 apart, u and h now and then take the neighbouring code
    model = MLP8(512, 1024, seed=5)
    x = torch.randn((40, 512), device="cuda").bfloat16()
    y = model.forward(x, keep=False)
    assert torch.equal(y, model.forward(x)[0])
    for i in (0, 17, 39):
        assert rel(model.forward(x[i:i + 1], keep=False), y[i:i + 1].double().cpu()) < 0.02


@pytest.mark.parametrize("tokens", [1, 24, 300])
def test_graph_replays(tokens):
    model = MLP8(512, 1024, seed=6)
    x = torch.randn((tokens, 512), device="cuda").bfloat16()
    dy = torch.randn((tokens, 512), device="cuda").bfloat16()
    side = torch.cuda.Stream()

    def step():
        y, kept = model.forward(x)
        dx, g = model.backward(dy, kept)
        return [y, dx, g["w1"], g["w2"], g["gamma"], g["beta"]]

    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()                                    # workspaces exist before the capture
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = step()
    for i in range(4):
        x.copy_(torch.randn_like(x))
        dy.copy_(torch.randn_like(dy))
        want = step()
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
