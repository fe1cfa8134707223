"""The routed layer on a stream that is not torch's current one: inputs that are still being made, results that are used at once and memory that
is handed on, all without a synchronisation of the caller's."""
import pytest
import torch

from paper_2310_18859_amd import streams_create, streams_destroy
from paper_2310_18859_amd.mx_layer import MxMoELayer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
T, E, D, F, K = 300, 8, 256, 384, 2


def busy():
    """Some milliseconds of work on the current stream."""
    a = torch.full((4096, 4096), 1e-3, device=DEV)
    for _ in range(8):
        a = a @ a
    return a


def inputs(seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    return dict(w_in=normal(E, F, D).mul_(0.08).bfloat16(), w_out=normal(E, D, F).mul_(0.08).bfloat16(), x=normal(T, D).bfloat16(), logits=normal(T, E) * 2,
                mask=torch.rand(T, generator=g, device=DEV) < 0.9, dy=normal(T, D).bfloat16(), d_loss=torch.tensor([0.01], device=DEV))


def results(layer, v, late):
    """What the layer makes of v, taken on the current stream right behind the calls.  late: each call's inputs are written behind other
    work of the current stream, and once a call has returned their memory is given away and written over."""
    def given(name):
        if not late:
            return v[name]
        t = torch.zeros_like(v[name])
        t.copy_(v[name])
        return t

    def over(*names):
        for n in names:
            torch.full_like(v[n], float("nan") if v[n].is_floating_point() else 0)

    if late:
        busy()
    w = given("w_in"), given("w_out").transpose(1, 2).contiguous().transpose(1, 2)     # the second is copied within the call
    layer.load_experts(*w)
    del w
    over("w_in", "w_out")
    if late:
        busy()
    x, logits, mask = given("x"), given("logits"), given("mask")
    y, loss = layer.forward(x, logits, mask)
    del x
    over("x", "x")
    out = [y.clone(), loss.clone(), layer.ids[:T].clone(), layer.gates[:T].clone(), layer.counts.clone()]
    del y
    over("x", "x")
    if late:
        busy()
    dy, d_loss = given("dy"), given("d_loss")
    grad = layer.router_gradient(logits, dy, d_loss, mask)
    del dy, d_loss, logits, mask
    over("dy", "logits", "logits")
    out.append(grad.clone())
    return out


@pytest.fixture(scope="module")
def want():
    v = inputs(1)
    layer = MxMoELayer(E, D, F, T, top_k=K, normalize=True)
    out = results(layer, v, False)
    torch.cuda.synchronize()
    layer.close()
    return v, out


@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("way", ["given", "raw", "raw null", "made outside", "made inside"])
def test_other_streams(want, way, x4):
    v, expected = want
    side = torch.cuda.Stream()
    raw = streams_create(0) if way == "raw" else None
    args = dict(top_k=K, normalize=True, tokens_in_4_bits=x4)
    called = torch.cuda.current_stream()
    if way == "given":
        layer = MxMoELayer(E, D, F, T, stream=side, **args)
    elif way == "raw":
        layer = MxMoELayer(E, D, F, T, stream=raw[0], **args)
    elif way == "raw null":
        layer, called = MxMoELayer(E, D, F, T, stream=0, **args), side
    elif way == "made outside":
        layer, called = MxMoELayer(E, D, F, T, **args), side
    else:
        with torch.cuda.stream(side):
            layer = MxMoELayer(E, D, F, T, **args)
    torch.cuda.synchronize()
    if x4:                                                             # what the same layer gives on one stream
        one = MxMoELayer(E, D, F, T, **args)
        expected = results(one, v, False)
        torch.cuda.synchronize()
        one.close()
    with torch.cuda.stream(called):
        for _ in range(3):
            with torch.cuda.stream(layer.stream):
                busy()                                                 # the layer's stream is behind as well
            for got, w in zip(results(layer, v, True), expected):
                assert torch.equal(got, w)
    torch.cuda.synchronize()
    layer.close()
    if raw:
        del layer
        torch.cuda.empty_cache()
        streams_destroy(*raw)


def test_strided_and_shifted_tokens(want):
    """Rows with something between them, columns in another order and rows off a 16-byte boundary give what packed rows give."""
    v, expected = want
    layer = MxMoELayer(E, D, F, T, top_k=K, normalize=True)
    layer.load_experts(v["w_in"], v["w_out"])
    wide = torch.full((T, D + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
    wide[:, 8:] = v["x"]
    shifted = torch.full((T * D + 1,), float("nan"), dtype=torch.bfloat16, device=DEV)[1:].view(T, D)
    shifted.copy_(v["x"])
    for x in (wide[:, 8:], v["x"].t().contiguous().t(), shifted):
        y, _ = layer.forward(x, v["logits"], v["mask"])
        assert y.is_contiguous() and torch.equal(y, expected[0])
    layer.close()
