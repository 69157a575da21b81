"""One pre-norm MLP block, y = x + W2 gelu(W1 norm(x)), trained and served on the 8-bit path.

    python examples/mlp8.py [--d 512] [--ffn 2048] [--tokens 2048] [--steps 200] [--sparse] [--rms] [--fused]

Forward: the norm writes its result in 8 bits, which is at once the product's operand and all of it that is kept for the
backward; so are gelu's input and output, and the block's input for the norm's gradient: 2 d + 2 ffn bytes a token instead
of 4 d + 4 ffn in bf16. Backward: the input gradients are the same product on the transposed packs, the weight gradients
take the kept 8-bit rows as they are, and the norm's gradient its 8-bit input. With --sparse W2 stays at its 2:4 positions:
its gradient is computed in compressed form, weight decay is the sparse add, and only kept values change. Master weights
are fp32; a step packs them anew. With --fused the products end in what follows them: gelu, its result and its argument in 8 bits
leave the first product's launch, the residual is added in the second's, and the gradient passes gelu in that of its own product.
"""
import argparse
import os
import sys
import time

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2608_24070_amd import slim  # noqa: E402


class MLP8:
    def __init__(self, d: int, ffn: int, sparse: bool = False, rms: bool = False, seed: int = 0, device="cuda",
                 fused: bool = False):
        g = torch.Generator(device).manual_seed(seed)
        rand = lambda n, k: torch.randn((n, k), generator=g, device=device) * k ** -0.5
        self.w1, self.w2 = rand(ffn, d), rand(d, ffn)
        self.gamma = torch.ones(d, device=device)
        self.beta = None if rms else torch.zeros(d, device=device)
        self.rms, self.values, self.fused = rms, None, fused
        if sparse:
            self.values = slim.pack16(self.w2, with_mask=True)
            self.kept = self.values["mask"].bool()
            self.w2 *= self.kept
        self.pack()

    def pack(self):
        self.p1, self.p2 = slim.pack8(self.w1, bwd=True), slim.pack8(self.w2, bwd=True)

    def forward(self, x, keep: bool = True):
        """y for x [tokens, d] in bf16, and with `keep` what the backward needs."""
        n, mean, rstd = slim.norm(x, self.gamma, self.beta, rms=self.rms, q8=True)
        if self.fused:
            return self._forward_fused(x, n, mean, rstd, keep)
        u = slim.linear8(n, self.p1)
        h = F.gelu(u)
        if not keep:
            return x + slim.linear8(h, self.p2)
        h = slim.quant8(h)
        return x + slim.linear8(h, self.p2), {"x": slim.quant8(x), "mean": mean, "rstd": rstd, "n": n, "u": slim.quant8(u), "h": h}

    def _forward_fused(self, x, n, mean, rstd, keep):
        if not keep:
            return slim.linear8_act(slim.linear8_act(n, self.p1, act="gelu"), self.p2, residual=x)
        h, u = slim.linear8_act(n, self.p1, act="gelu", pre=True, q8=True)
        y = slim.linear8_act(h, self.p2, residual=x)
        return y, {"x": slim.quant8(x), "mean": mean, "rstd": rstd, "n": n, "u": u, "h": h}

    def backward(self, dy, kept):
        """dx and the gradients of the weights (W2's at its kept positions, if it is sparse), gamma and beta."""
        if self.fused:
            du, _, _ = slim.bwd_dx8_act(dy, self.p2, kept["u"], act="gelu", dtype=dy.dtype)
        else:
            du = torch.ops.aten.gelu_backward(slim.bwd_dx8(dy, self.p2), slim.dequant8(kept["u"], dy.dtype))
        g = {"w2": slim.grad_w8(dy, kept["h"], self.values), "w1": slim.grad_w8(du, kept["n"])}
        dx, g["gamma"], g["beta"] = slim.norm_bwd(slim.bwd_dx8(du, self.p1), kept["x"], self.gamma, kept["mean"], kept["rstd"])
        return dx + dy, g

    def step(self, g, lr: float, decay: float = 0.0):
        if self.values is None:
            self.w2.mul_(1 - lr * decay).sub_(g["w2"], alpha=lr)
        else:
            grad = slim.sparse_add(g["w2"], self.values["vals"], 1.0, decay)
            new = self.w2[self.kept].view_as(grad).sub_(grad, alpha=lr)
            slim.update_pack16(new, self.values)
            self.w2.masked_scatter_(self.kept, new)
        self.w1.mul_(1 - lr * decay).sub_(g["w1"], alpha=lr)
        self.gamma.sub_(g["gamma"], alpha=lr)
        if self.beta is not None:
            self.beta.sub_(g["beta"], alpha=lr)
        self.pack()


def kept_bytes(kept) -> int:
    tensors = [t for v in kept.values() for t in (v.values() if isinstance(v, dict) else [v])]
    return sum(t.numel() * t.element_size() for t in tensors if torch.is_tensor(t))


def train(model: MLP8, tokens: int, steps: int, lr: float, decay: float = 0.0, seed: int = 1):
    """Mean squared errors per step against a fixed random linear map of the input."""
    d = model.gamma.numel()
    g = torch.Generator(model.gamma.device).manual_seed(seed)
    teacher = torch.randn((d, d), generator=g, device=model.gamma.device) * d ** -0.5
    losses = []
    for _ in range(steps):
        x = torch.randn((tokens, d), generator=g, device=model.gamma.device).bfloat16()
        y, kept = model.forward(x)
        diff = y.float() - (x.float() @ teacher)
        losses.append(diff.square().mean())
        dx, grads = model.backward((diff * (2.0 / tokens)).bfloat16(), kept)
        model.step(grads, lr, decay)
    return [float(v) for v in losses]


def main():
    a = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    a.add_argument("--d", type=int, default=512)
    a.add_argument("--ffn", type=int, default=2048)
    a.add_argument("--tokens", type=int, default=2048)
    a.add_argument("--steps", type=int, default=200)
    a.add_argument("--lr", type=float, default=0.01)
    a.add_argument("--decay", type=float, default=0.0)
    a.add_argument("--sparse", action="store_true", help="W2 at 2:4 positions (d and ffn in whole 128s)")
    a.add_argument("--rms", action="store_true", help="RMS norm instead of layer norm")
    a.add_argument("--fused", action="store_true", help="products that end in the activation and the residual")
    a = a.parse_args()
    model = MLP8(a.d, a.ffn, a.sparse, a.rms, fused=a.fused)
    train(MLP8(a.d, a.ffn, a.sparse, a.rms, fused=a.fused), a.tokens, 2, a.lr, a.decay)
    torch.cuda.synchronize()
    t = time.time()
    losses = train(model, a.tokens, a.steps, a.lr, a.decay)
    torch.cuda.synchronize()
    t = time.time() - t
    x = torch.randn((a.tokens, a.d), device="cuda").bfloat16()
    _, kept = model.forward(x)
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f} over {a.steps} steps, {a.tokens * a.steps / t:.0f} tokens/s")
    print(f"kept for the backward: {kept_bytes(kept) / a.tokens:.0f} bytes a token ({4 * a.d + 4 * a.ffn} in bf16)")
    # single tokens, captured once and replayed
    one = x[:1].clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())      # for `one` and the weights
    with torch.cuda.stream(side):
        model.forward(one, keep=False)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        y = model.forward(one, keep=False)
    graph.replay()
    start, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    start.record()
    for _ in range(100):
        graph.replay()
    end.record()
    torch.cuda.synchronize()
    print(f"one token: {start.elapsed_time(end) * 10:.1f} us, |y| {float(y.float().norm()):.3f}")


if __name__ == "__main__":
    main()
