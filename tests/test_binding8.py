"""What the binding of the 8-bit path refuses before it makes a pointer of it; no call here reaches a device."""
import pytest
import torch

from paper_2608_24070_amd import slim


class Reached(Exception):
    """A call got past its checks."""


@pytest.fixture
def on_gpu(monkeypatch):
    """Host tensors pass for device ones; the check that follows the types' ends the call."""
    def reached(*ts):
        raise Reached
    monkeypatch.setattr(slim, "_on_gpu", reached)
    monkeypatch.setattr(slim, "_matrix", lambda t, what: (t.shape[0], t.shape[1], t.shape[1], t.get_device()))


def rows8(m=4, k=256, codes=torch.uint8, exps=torch.uint8):
    return {"codes": torch.zeros((m, k), dtype=codes), "exps": torch.zeros((m, 4), dtype=exps), "M": m, "K": k}


def weight8(n=32, k=256, codes=torch.uint8, exps=torch.uint8):
    c, e = torch.zeros((n // 16, k // 128, 2, 4, 16, 16), dtype=codes), torch.zeros((1, 4), dtype=exps)
    return {"codes": c, "exps": e, "codesT": c, "expsT": e, "N": n, "K": k}


WRONG = [dict(codes=torch.float8_e4m3fn), dict(codes=torch.float32), dict(codes=torch.int16), dict(exps=torch.int32), dict(exps=torch.float32)]


@pytest.mark.parametrize("kw", WRONG)
def test_codes_and_exponents_are_bytes(on_gpu, kw):
    x = torch.zeros((4, 256), dtype=torch.bfloat16)
    dy = torch.zeros((4, 32), dtype=torch.bfloat16)
    s = torch.zeros(4)
    # each call's first operand in 8 bits: of bytes it passes, of anything else it does not
    calls = [lambda r, w: slim.dequant8(r), lambda r, w: slim.linear8(x, w), lambda r, w: slim.quant8(x, out=r),
             lambda r, w: slim.bwd_dx8(x, dict(w, N=256, K=32)), lambda r, w: slim.norm(x, q8=True, out=r),
             lambda r, w: slim.grad_w8(dy, r), lambda r, w: slim.norm_bwd(x, r, None, s, s)]
    for call in calls:
        with pytest.raises(Reached):
            call(rows8(), weight8())
        with pytest.raises(TypeError, match="uint8"):
            call(rows8(**kw), weight8(**kw))


class OnGpu(torch.Tensor):
    """A host tensor that says it is on a device."""
    is_cuda = True

    def get_device(self):
        return 0


def test_a_given_workspace_is_device_memory_of_its_size():
    gpu = lambda t: t.as_subclass(OnGpu)
    like = gpu(torch.zeros(1))
    ws = gpu(torch.zeros(4096, dtype=torch.uint8))
    assert slim._given8(4000, ws, like, 0) == (ws.data_ptr(), 4096)
    assert slim._given8(0, None, like, 0) == (None, 0)
    wide = gpu(torch.zeros(1024))
    assert slim._given8(4000, wide, like, 0) == (wide.data_ptr(), 4096)
    for bad in (torch.zeros(4096, dtype=torch.uint8),                  # on the host
                gpu(torch.zeros(1, dtype=torch.uint8)).expand(4096),   # one byte
                gpu(torch.zeros(8192, dtype=torch.uint8))[::2]):
        with pytest.raises(ValueError):
            slim._given8(4000, bad, like, 0)


class Elsewhere(OnGpu):
    def get_device(self):
        return 1


def test_a_given_workspace_is_on_the_tensors_device():
    with pytest.raises(ValueError, match="device"):
        slim._given8(10, torch.zeros(4096, dtype=torch.uint8).as_subclass(Elsewhere), torch.zeros(1).as_subclass(OnGpu), 0)


def test_the_compressed_layer_looks_at_its_workspace_too(monkeypatch):
    seen = []

    def record(*ts):
        seen.extend(ts)
        raise Reached

    monkeypatch.setattr(slim, "_on_gpu", record)
    x, ws = torch.zeros((4, 256), dtype=torch.bfloat16), torch.zeros(8)
    for call in (lambda: slim.linear(x, {"N": 32}, ws=ws), lambda: slim.bwd_dx(x, {"K": 32}, ws=ws),
                 lambda: slim.linear_qa(x, {"N": 32}, {"r": 32}, ws=ws)):
        seen.clear()
        with pytest.raises(Reached):
            call()
        assert any(t is ws for t in seen)
