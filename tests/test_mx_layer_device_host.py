"""The routed layer makes its device the current one for what it does there: the library launches on the current device.  Checked with stand-ins for
torch's device and streams (one GPU cannot tell), and on a second GPU where there is one."""
import contextlib

import pytest
import torch

from paper_2310_18859_amd import mx_layer


class Stream:
    def __init__(self):
        self.waited = []

    def wait_stream(self, other):
        self.waited.append(other)


@pytest.mark.parametrize("own", [False, True])
def test_the_layers_device_is_current(monkeypatch, own):
    now = [0]                                                          # the current device, of two

    @contextlib.contextmanager
    def device(d):
        before, now[0] = now[0], torch.device(d).index
        try:
            yield
        finally:
            now[0] = before

    @contextlib.contextmanager
    def stream(s):                                                     # does not set the device here
        yield

    current = Stream()
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda d=None: current)
    layer = mx_layer.MxMoELayer.__new__(mx_layer.MxMoELayer)
    layer.dev, layer.stream = torch.device("cuda:1"), Stream() if own else current
    with layer._on_stream():
        assert now == [1]
        assert not own or (layer.stream.waited == [current] and not current.waited)
    assert now == [0]
    assert not own or current.waited == [layer.stream]
    with pytest.raises(ZeroDivisionError), layer._on_stream():
        1 / 0
    assert not own or current.waited == [layer.stream] * 2             # also after an error


@pytest.mark.gpu
@pytest.mark.skipif(torch.cuda.device_count() < 2, reason="needs a second GPU")
def test_layer_on_a_second_gpu():
    results = []
    for d in ("cuda:0", "cuda:1"):
        g = torch.Generator().manual_seed(1)
        w_in, w_out, x, logits, dy = (torch.randn(s, generator=g).to(d) for s in ((4, 256, 128), (4, 128, 256), (50, 128), (50, 4), (50, 128)))
        layer = mx_layer.MxMoELayer(4, 128, 256, 50, top_k=2, device=d)
        layer.load_experts(w_in, w_out)
        y, loss = layer.forward(x.bfloat16(), logits)
        grad = layer.router_gradient(logits, dy, torch.ones(1, device=d))
        results.append([t.cpu() for t in (y, loss, grad)])
        layer.close()
    assert all(torch.equal(a, b) for a, b in zip(*results))
