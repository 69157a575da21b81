"""The 8-bit helpers on a stream that is given: what they allocate belongs to it, and it must be of the tensors' device."""
import threading

import pytest
import torch

from paper_2608_24070_amd import slim

pytestmark = pytest.mark.gpu


def stream_of(t):
    """The stream on which the allocator handed out t's memory."""
    for segment in torch.cuda.memory_snapshot():
        if segment["address"] <= t.data_ptr() < segment["address"] + segment["total_size"]:
            return segment["stream"]


def tensors(r):
    if torch.is_tensor(r):
        return [r]
    return [t for v in (r.values() if isinstance(r, dict) else r if isinstance(r, tuple) else ()) for t in tensors(v)]


def test_results_belong_to_the_given_stream():
    x = torch.randn((300, 640), device="cuda").bfloat16()
    dy = torch.randn((300, 256), device="cuda").bfloat16()
    w = torch.randn((256, 640), device="cuda")
    gamma = torch.ones(640, device="cuda")
    q, p = slim.quant8(x), slim.pack8(w, bwd=True)
    y, mean, rstd = slim.norm(x, gamma)
    calls = {"quant8": lambda **k: slim.quant8(x, **k), "dequant8": lambda **k: slim.dequant8(q, **k),
             "pack8": lambda **k: slim.pack8(w, bwd=True, **k), "linear8": lambda **k: slim.linear8(x, p, **k),
             "bwd_dx8": lambda **k: slim.bwd_dx8(dy, p, **k), "grad_w8": lambda **k: slim.grad_w8(dy, q, **k),
             "norm": lambda **k: slim.norm(x, gamma, **k), "norm to 8 bits": lambda **k: slim.norm(x, gamma, q8=True, **k),
             "norm_bwd": lambda **k: slim.norm_bwd(x, q, gamma, mean, rstd, **k)}
    here = torch.cuda.current_stream()
    for name, call in calls.items():
        want = tensors(call())
        s = torch.cuda.Stream()
        s.wait_stream(here)
        got = tensors(call(stream=s))
        assert torch.cuda.current_stream() == here
        s.synchronize()
        assert len(got) == len(want) > 0
        for a, b in zip(got, want):
            assert stream_of(a) == s.cuda_stream and torch.equal(a, b), name


def test_a_tensor_elsewhere_is_refused():
    with pytest.raises(ValueError, match="device"):
        slim.quant8(torch.zeros((2, 128)), stream=torch.cuda.Stream())


def test_threads_on_one_stream_keep_apart():
    # rows that are quantised into the workspace before the product: no thread may fill it between another's two launches
    p = slim.pack8(torch.randn((256, 640), device="cuda"))
    xs = [torch.randn((40, 640), device="cuda").bfloat16() for _ in range(4)]
    want = [slim.linear8(x, p) for x in xs]
    torch.cuda.synchronize()
    wrong = []

    def work(i):
        wrong.extend(j for j in range(200) if not torch.equal(slim.linear8(xs[i], p), want[i]))

    threads = [threading.Thread(target=work, args=(i,)) for i in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
