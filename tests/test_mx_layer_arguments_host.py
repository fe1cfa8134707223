"""What the routed layer refuses before anything is enqueued, and what it lets through: no GPU is needed."""
import contextlib

import pytest
import torch

from paper_2310_18859_amd import mx_layer

E, D, F, K, T = 4, 128, 256, 2, 6
BF16, FP32 = torch.bfloat16, torch.float32


class Reached(Exception):
    pass


@pytest.fixture
def layer(monkeypatch):
    """A layer on the CPU whose way to the library ends where its stream would be taken."""
    @contextlib.contextmanager
    def reached(self, *_):
        raise Reached
        yield

    monkeypatch.setattr(mx_layer.MxMoELayer, "_on_stream", reached, raising=False)
    made = mx_layer.MxMoELayer.__new__(mx_layer.MxMoELayer)
    made.__dict__.update(E=E, d=D, F=F, k=K, max_tokens=8, max_pairs=16, dev=torch.device("cpu"), loaded=True, tokens=T, x4=False, normalize=False,
                         ids=None, gates=None, counts=None, loss=None, stream=None, ctx=None)
    return made


def x(rows=T, cols=D, dtype=BF16, **kw):
    return torch.zeros((rows, cols), dtype=dtype, **kw)


@pytest.mark.parametrize("bad", [
    dict(x=x(dtype=FP32)), dict(x=x(dtype=torch.float16)),                    # taken for bf16
    dict(x=x(cols=64)), dict(x=x(cols=256)),                                  # rows of another width
    dict(x=torch.zeros(T * D, dtype=BF16)), dict(x=torch.zeros((2, 3, D), dtype=BF16)), dict(x=torch.zeros((), dtype=BF16)),
    dict(x=x(9), logits=x(9, E)),                                             # more tokens than there is room for
    dict(x=x(device="meta")), dict(logits=x(cols=E, device="meta")),
    dict(logits=x(T - 1, E)), dict(logits=x(T, E - 1)), dict(logits=x(T, E + 1)), dict(logits=x(T, E, torch.float16)),
])
def test_forward_refuses(layer, bad):
    with pytest.raises(ValueError):
        layer.forward(**{"x": x(), "logits": x(cols=E), **bad})


@pytest.mark.parametrize("good", [
    dict(), dict(logits=x(cols=E, dtype=FP32)), dict(x=x(8), logits=x(8, E)), dict(x=x(0), logits=x(0, E)),
    dict(x=x(cols=2 * D)[:, :D]), dict(x=x(D, T).t()), dict(x=torch.zeros(T * D + 1, dtype=BF16)[1:].view(T, D)),
])
def test_forward_lets_through(layer, good):
    with pytest.raises(Reached):
        layer.forward(**{"x": x(), "logits": x(cols=E), **good})


def test_forward_needs_experts(layer):
    layer.loaded = False
    with pytest.raises(RuntimeError):
        layer.forward(x(), x(cols=E))


def w(e=E, rows=F, cols=D, dtype=BF16, **kw):
    return torch.zeros((e, rows, cols), dtype=dtype, **kw)


@pytest.mark.parametrize("bad", [
    dict(w_in=w(E - 1)), dict(w_in=w(E + 1)), dict(w_out=w(E - 1, D, F)),     # the other experts would stay as they are
    dict(w_in=w(E, D, F)), dict(w_out=w()), dict(w_in=torch.zeros((E * F, D), dtype=BF16)), dict(w_out=w(E, D, F, torch.float16)),
    dict(w_in=w(device="meta")),
])
def test_load_experts_refuses(layer, bad):
    layer.loaded = False
    with pytest.raises(ValueError):
        layer.load_experts(**{"w_in": w(), "w_out": w(E, D, F), **bad})
    assert not layer.loaded


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_load_experts_lets_through(layer, dtype):
    with pytest.raises(Reached):
        layer.load_experts(w(dtype=dtype), w(E, D, F, dtype))


@pytest.mark.parametrize("bad", [
    dict(dy=x(1)), dict(dy=x(cols=1)), dict(dy=x(T - 1)), dict(dy=torch.zeros(D, dtype=BF16)),    # would be broadcast, or worse
    dict(logits=x(T - 1, E), dy=x(T - 1)), dict(logits=x(T, E + 1)), dict(dy=x(device="meta")), dict(dy=torch.zeros((T, D), dtype=torch.int32)),
])
def test_gradient_refuses(layer, bad):
    with pytest.raises(ValueError):
        layer.router_gradient(**{"logits": x(cols=E), "dy": x(), "d_loss": torch.zeros(1), **bad})


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_gradient_lets_through(layer, dtype):
    with pytest.raises(Reached):
        layer.router_gradient(x(cols=E, dtype=dtype), x(dtype=dtype), torch.zeros(()))
