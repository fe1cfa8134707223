"""What the layer that can be trained refuses by strides, alignment, masks and sizes, before anything is enqueued and with the last call's way back still there: no GPU is
needed."""
import contextlib

import pytest
import torch

from paper_2310_18859_amd import moe_layer

E, D, F, K, T = 4, 16, 24, 2, 6
BF16, FP32 = torch.bfloat16, torch.float32


class Reached(Exception):
    pass


def made(monkeypatch, **sizes):
    """A layer on the CPU whose way to the library ends where its stream would be taken."""
    @contextlib.contextmanager
    def reached(self, *_):
        raise Reached
        yield

    monkeypatch.setattr(moe_layer.MoELayer, "_on_stream", reached)
    layer = moe_layer.MoELayer.__new__(moe_layer.MoELayer)
    layer.__dict__.update(dict(E=E, d=D, F=F, k=K, act=2, max_tokens=8, dev=torch.device("cpu"), tokens=T, normalize=False, ids=None, gates=None, counts=None,
                               loss=None, stream=None), **sizes)
    return layer


def z(*shape, dtype=BF16, **kw):
    return torch.zeros(shape, dtype=dtype, **kw)


def off_by_one(*shape, dtype=BF16):
    """Contiguous, but not from a 16-byte boundary on."""
    n = 1
    for s in shape:
        n *= s
    return z(n + 1, dtype=dtype)[1:].view(shape)


GIVEN = dict(x=z(T, D), logits=z(T, E), w_in=z(E, F, D), w_out=z(E, D, F))
BACK = dict(dy=z(T, D), logits=z(T, E), w_in=z(E, F, D), w_out=z(E, D, F))
MASKS = [z(T, dtype=torch.float32), z(T, dtype=torch.int32), z(T - 1, dtype=torch.bool), z(2 * T, dtype=torch.bool)[::2], z(T, dtype=torch.bool, device="meta")]
WEIGHTS = [dict(w_in=off_by_one(E, F, D)), dict(w_out=off_by_one(E, D, F))]
LOGITS = [z(E, T).t(), z(T, 2 * E)[:, ::2], z(1, E).expand(T, E), z(E + T - 1).as_strided((T, E), (1, 1))]


@pytest.mark.parametrize("bad", [dict(x=z(D, T).t()), dict(x=z(T, 2 * D)[:, ::2]), dict(x=z(1, D).expand(T, D)), dict(residual=z(D, T).t()),
                                 dict(residual=z(1, D).expand(T, D)), dict(b_in=off_by_one(E, F, dtype=FP32)), dict(b_out=off_by_one(E, D, dtype=FP32))]
                         + WEIGHTS + [dict(logits=t) for t in LOGITS] + [dict(mask=m) for m in MASKS])
def test_forward(monkeypatch, bad):
    layer = made(monkeypatch)
    with pytest.raises(ValueError):
        layer.forward(**{**GIVEN, **bad})
    assert layer.tokens == T                                            # the last call's way back is still there


@pytest.mark.parametrize("good", [dict(mask=z(T, dtype=torch.bool)), dict(mask=z(T + 3, dtype=torch.uint8)), dict(logits=z(T, 2 * E)[:, :E]),
                                  dict(x=z(1, 2 * D)[:, :D], logits=z(1, E)), dict(x=z(0, D), logits=z(0, E), residual=z(0, D)), dict(x=off_by_one(T, D)),
                                  dict(residual=z(T, D + 3)[:, 3:])])
def test_forward_lets_through(monkeypatch, good):
    with pytest.raises(Reached):
        made(monkeypatch).forward(**{**GIVEN, **good})


@pytest.mark.parametrize("bad", [dict(dy=z(D, T).t()), dict(dy=z(1, 1).expand(T, D)), dict(d_loss=z(1)), dict(d_loss=z(0, dtype=FP32)),
                                 dict(d_loss=z(1, dtype=FP32, device="meta"))] + WEIGHTS + [dict(logits=t) for t in LOGITS] + [dict(mask=m) for m in MASKS])
def test_backward(monkeypatch, bad):
    with pytest.raises(ValueError):
        made(monkeypatch).backward(**{**BACK, **bad})


@pytest.mark.parametrize("good", [dict(d_loss=z(1, dtype=FP32), mask=z(T, dtype=torch.bool)), dict(d_loss=torch.zeros(())),
                                  dict(dy=z(T, 2 * D)[:, D:]), dict(biases=False)])
def test_backward_lets_through(monkeypatch, good):
    with pytest.raises(Reached):
        made(monkeypatch).backward(**{**BACK, **good})


@pytest.mark.parametrize("k,d,F_,tokens", [(8, 8, 8, (1 << 21) + 1), (1, 8, 65536, (1 << 19) + 1), (1, 65536, 8, (1 << 19) + 1), (2, 4096, 16384, (1 << 20) + 1)])
def test_more_pairs_than_the_products_take(monkeypatch, k, d, F_, tokens):
    """Pairs up to 2^24, and pairs times width up to 2^35."""
    layer = made(monkeypatch, k=k, d=d, F=F_, max_tokens=1 << 30)
    for T, raised in ((tokens, ValueError), (tokens - 1, Reached)):
        meta = dict(dtype=BF16, device="meta")
        layer.dev, layer.tokens = torch.device("meta"), 5
        with pytest.raises(raised):
            layer.forward(torch.empty((T, d), **meta), torch.empty((T, E), **meta), torch.empty((E, F_, d), **meta), torch.empty((E, d, F_), **meta))
        assert layer.tokens == (5 if raised is ValueError else None)


@pytest.mark.parametrize("bad", [dict(E=0), dict(E=257), dict(top_k=0), dict(top_k=9, E=16), dict(top_k=5), dict(d_model=0), dict(d_ff=0), dict(d_model=65544),
                                 dict(d_ff=65544), dict(d_model=32768, d_ff=32776), dict(E=256, d_model=16384, d_ff=16392), dict(max_tokens=-1), dict(max_tokens=1 << 25, top_k=2)])
def test_sizes_refused(bad):
    with pytest.raises(ValueError):
        moe_layer.MoELayer(**{"E": E, "d_model": D, "d_ff": F, "max_tokens": 8, **bad})
