"""The memory that a captured call's kernels write is its graph's for as long as the graph lives. The binding's kept workspaces
are not: a larger call replaces them, and a thread takes its own with it. Here with host tensors in the place of device ones
and a stream that says it is captured (no kernel runs)."""
import pytest
import torch

from paper_2608_24070_amd import slim

STREAM = 7          # a handle nobody uses


@pytest.fixture
def capture(monkeypatch):
    """capture(True): from here on the stream is being captured."""
    state = [False]
    monkeypatch.setattr(slim, "_capturing", lambda dev: state[0], raising=False)
    return lambda on: state.__setitem__(0, on)


def overlap(a, b):
    return a.data_ptr() < b.data_ptr() + b.numel() and b.data_ptr() < a.data_ptr() + a.numel()


def test_the_8_bit_calls(capture):
    like = torch.empty(0, dtype=torch.uint8)
    kept = slim._workspace8(1000, like, STREAM)
    assert slim._workspace8(500, like, STREAM) is kept
    capture(True)
    mine = slim._workspace8(1000, like, STREAM)
    assert mine.numel() >= 1000 and not overlap(mine, kept)
    larger = slim._workspace8(1 << 20, like, STREAM)
    assert larger.numel() >= 1 << 20 and not overlap(larger, mine)
    capture(False)
    # nothing of the capture is kept, and what was kept before it still is
    assert slim._workspace8(1000, like, STREAM) is kept
    grown = slim._workspace8(1 << 20, like, STREAM)
    assert not any(overlap(grown, t) for t in (mine, larger))


def test_the_compressed_layer(capture, monkeypatch):
    monkeypatch.setattr(slim, "_stream", lambda stream=None: STREAM)
    monkeypatch.setattr(slim, "_ws_cache", {})
    kept = slim.workspace(100000, "cpu")
    assert slim.workspace(70000, "cpu") is kept and not kept.any()
    kept[0] = 1
    capture(True)
    mine = slim.workspace(100000, "cpu")
    assert mine.numel() >= 100000 and not overlap(mine, kept)
    assert not mine[:4096 * 4].any()          # the control words start at zero
    assert slim.workspace(100, "cpu").numel() >= 4096 * 4
    capture(False)
    assert slim.workspace(100000, "cpu") is kept
    grown = slim.workspace(1 << 20, "cpu")
    assert not overlap(grown, mine) and not grown.any()


def test_the_hybrid_layer(capture, monkeypatch):
    dev = torch.device("cpu")
    sizes = []

    def call(nbytes):
        """The workspace that linear_hybrid takes for a call that needs nbytes."""
        given = []
        monkeypatch.setattr(slim, "slim_linear_hybrid_workspace", lambda M, N, K: nbytes)
        monkeypatch.setattr(slim, "slim_linear_hybrid", lambda *a: given.append((a[8], a[9])) or slim.SLIM_OK)
        slim.linear_hybrid(x, {"N": 128, "K": 128, "tile_info": x, "payload": x})
        sizes.append(given[0][1])
        return given[0][0]

    monkeypatch.setattr(slim, "_on_gpu", lambda *ts: None)
    monkeypatch.setattr(slim, "_stream", lambda stream=None: STREAM)
    monkeypatch.setattr(slim, "_hybrid_ws", {})
    x = torch.zeros((2, 128), dtype=torch.float16)
    kept = call(1000)
    assert call(1000) == kept == slim._hybrid_ws[(dev, STREAM)].data_ptr()
    capture(True)
    assert call(1000) != kept
    call(1 << 20)
    capture(False)
    assert call(1000) == kept == slim._hybrid_ws[(dev, STREAM)].data_ptr()
    assert sizes == [1000, 1000, 1000, 1 << 20, 1000]
