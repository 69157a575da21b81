"""The example's block with products that end in its activation and residual, against the block in 64 bits: the bound, and why, as in
the tests of the block without them (the roundings to 8 bits are the same ones)."""
import pytest
import torch

from examples.mlp8 import MLP8, kept_bytes, train
from paper_2608_24070_amd import slim
from tests.gpu_common import kernels_of
from tests.test_gpu_mlp8 import ROUNDED, block, rel

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,d,ffn", [(1, 128, 256), (33, 256, 384), (500, 512, 1408)])
@pytest.mark.parametrize("rms", [False, True])
@pytest.mark.parametrize("sparse", [False, True])
def test_against_64_bits(tokens, d, ffn, rms, sparse):
    model = MLP8(d, ffn, sparse, rms, seed=3, fused=True)
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
    # what is kept is what the block without them keeps
    words = lambda k: -(-k // 512) * 4
    assert kept_bytes(kept) == tokens * (2 * (d + words(d)) + 2 * (ffn + words(ffn)) + 4 * (1 if rms else 2))
    assert rel(model.forward(x, keep=False), y.double().cpu()) < 0.02


def test_training_runs_and_one_token_is_few_launches():
    model = MLP8(256, 512, fused=True)
    assert all(v == v for v in train(model, 512, 3, lr=0.01))
    x = torch.randn((1, 256), device="cuda").bfloat16()
    assert kernels_of(lambda: model.forward(x, keep=False)) <= {"norm", "act8_few"}


@pytest.mark.parametrize("tokens", [1, 24, 300])
def test_graph_replays(tokens):
    model = MLP8(512, 1024, seed=6, fused=True)
    x = torch.randn((tokens, 512), device="cuda").bfloat16()
    dy = torch.randn((tokens, 512), device="cuda").bfloat16()

    def step():
        y, kept = model.forward(x)
        dx, g = model.backward(dy, kept)
        return [y, dx, g["w1"], g["w2"], g["gamma"], g["beta"], model.forward(x, keep=False)]

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for i in range(3):
        x.normal_()
        dy.normal_()
        want = step()
        for t in got:
            t.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want)), i
