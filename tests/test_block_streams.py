"""Waves of a block and its evaluation called under streams other than the session's: everything that touches rings and gradients goes to the
session's stream, in order with the caller's."""
import pytest
import torch

from paper_1902_01064_amd import block as bl
from paper_1902_01064_amd import hop, inputs, layers

pytestmark = pytest.mark.gpu


def training():
    block = bl.ResidualBlock(32, 48, p=0.1)
    data, held = bl.teacher_data(block, 5, 200, 3)
    return bl.Training(block, inputs.ring(5), data, 12, batch=20, lr=8.0, seed=11), held


def test_every_call_of_a_wave_is_on_the_sessions_stream(monkeypatch):
    t, held = training()
    seen = []

    def watched(module, name):
        call = getattr(module, name)

        def wrapper(*a, **k):
            seen.append((name, torch.cuda.current_stream().cuda_stream))
            return call(*a, **k)
        monkeypatch.setattr(module, name, wrapper)
    for name in ("norm", "product", "dropout", "residual", "residual_grad", "product_grad", "norm_grad"):
        watched(layers, name)
    watched(hop, "hop_step")
    try:
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            t.wave(0)
            t.evaluate(*held)
            assert torch.cuda.current_stream() == side
        torch.cuda.synchronize()
        assert {name for name, _ in seen} == {"norm", "product", "dropout", "residual", "residual_grad", "product_grad", "norm_grad", "hop_step"}
        assert {stream for _, stream in seen} == {t.session.stream} and side.cuda_stream != t.session.stream
    finally:
        t.close()


def run(under):
    """Losses and rings of a whole run; under(i): the stream that call i is made on."""
    t, held = training()
    losses, calls = [], 0
    busy = torch.randn(2048, 2048, device="cuda")
    try:
        for w in range(t.schedule.n_waves):
            for call in (lambda: t.wave(w), lambda: t.evaluate(*held).mean()):
                with torch.cuda.stream(under(calls, t)):
                    for _ in range(calls % 3):
                        busy = torch.tanh(busy @ busy)                  # work that the call has to stand behind
                    loss = call()
                    losses.append(None if loss is None else float(loss))
                calls += 1
        torch.cuda.synchronize()
        return losses, t.session.ring_snapshot()
    finally:
        t.close()


def test_the_callers_stream_does_not_matter():
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    want, rings = run(lambda i, t: t.stream)
    got, other = run(lambda i, t: (streams + [t.stream])[i % 3])
    assert want == got and (rings == other).all()
    with torch.cuda.stream(streams[0]):                                 # a session on a stream of its own
        got, other = run(lambda i, t: (streams + [torch.cuda.default_stream()])[i % 3])
    assert want == got and (rings == other).all()
