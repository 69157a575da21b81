"""The example's captured part on the host: streams, graph and model are stand-ins that write down what happens in which order."""
import contextlib

import torch

from examples import mlp8


def test_the_side_stream_waits_for_what_it_reads(monkeypatch, capsys):
    log, current = [], ["main"]

    class Stream:
        cuda_stream = 1

        def wait_stream(self, other):
            log.append(("side waits for", other))

        def synchronize(self):
            log.append(("synchronize", "side"))

    @contextlib.contextmanager
    def on(stream, name):
        before, current[0] = current[0], name
        yield
        current[0] = before

    class Graph:
        def replay(self):
            log.append(("replay", current[0]))

    class Event:
        def __init__(self, **kw):
            pass

        def record(self):
            pass

        def elapsed_time(self, other):
            return 1.0

    class Model:
        def __init__(self, *a, **kw):
            pass

        def forward(self, x, keep=True):
            log.append(("forward", current[0]))
            return (x, {}) if keep else x

    randn = torch.randn
    monkeypatch.setattr(torch, "randn", lambda *a, device=None, **kw: randn(*a, **kw))
    monkeypatch.setattr(mlp8, "MLP8", Model)
    monkeypatch.setattr(mlp8, "train", lambda *a, **kw: [1.0, 0.5])
    monkeypatch.setattr(mlp8.sys, "argv", ["mlp8.py", "--d", "8", "--tokens", "4"])
    for name, fake in (("Stream", Stream), ("stream", lambda s: on(s, "side")), ("graph", lambda g, stream=None: on(stream, "side")), ("CUDAGraph", Graph),
                       ("Event", Event), ("synchronize", lambda: None), ("current_stream", lambda *a: current[0])):
        monkeypatch.setattr(torch.cuda, name, fake)
    mlp8.main()
    assert "one token" in capsys.readouterr().out
    assert ("side waits for", "main") in log
    assert log.index(("side waits for", "main")) < log.index(("forward", "side")) < log.index(("replay", "main"))
