"""The routed layer that can be trained: forward and backward as one run of its operators, against the definitions in 64 bits and against differences.

Tolerances: what the layer keeps in bf16 (the hidden values, what is in front of them, the experts' outputs, their gradients) is off by half a step, 2^-8, of the
value each time it is rounded; the comparison rounds at the same places in 64 bits, so that only the sums' own errors, and values on the other side of a
rounding's border, remain: a step of bf16 of the largest magnitude of the tensor, 2^-7, on each value, and 2^-8 of the norm on all."""
import math

import pytest
import torch

import paper_2310_18859_amd as sm
from oracle import experts as plain
from paper_2310_18859_amd.moe_layer import ACTIVATIONS, MoELayer

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32


def bf(t):
    return t.to(BF).double()


def make(T, E, d, F, k, seed=0, masked=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g)  # noqa: E731
    v = dict(x=r(T, d).to(BF), logits=r(T, E) * 2, w_in=(r(E, F, d) / math.sqrt(d)).to(BF), w_out=(r(E, d, F) / math.sqrt(F)).to(BF), b_in=r(E, F) * 0.1,
             b_out=r(E, d) * 0.1, residual=r(T, d).to(BF), dy=r(T, d).to(BF), d_loss=torch.tensor([0.5]))
    v["mask"] = torch.rand(T, generator=g) < 0.8 if masked else None
    if masked and T > 3:
        v["logits"][2] = -float("inf")                                 # takes no part, either
        v["x"][2] = float("nan")
    return v


def chosen(v, k, normalize):
    """(ids, gates, part) of the router's definition."""
    z = v["logits"].double()
    part = ~torch.isinf(z).all(1)
    if v["mask"] is not None:
        part &= v["mask"]
    p = torch.softmax(z, 1)
    ids = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    gates = torch.gather(p, 1, ids)
    if normalize:
        gates = gates / gates.sum(1, keepdim=True)
    return ids, torch.where(part[:, None], gates, 0.0), part


def reference(v, E, d, F, k, act, normalize, biases, residual):
    T = v["x"].shape[0]
    ids, gates, part = chosen(v, k, normalize)
    gates = gates.float()
    offsets, places = plain.sort(torch.where(part[:, None], ids, -1), gates, E)
    at = offsets.tolist()
    n = at[-1]
    group = torch.bucketize(torch.arange(n), offsets[1:].long(), right=True)
    xr = plain.rows(v["x"], places, torch.zeros(n, d))
    pre = plain.product(xr, v["w_in"], at)[0]
    pre = pre + (v["b_in"].double()[group] if biases else 0)
    h = bf(plain.activation(pre, act))
    yr = plain.product(h, v["w_out"], at)[0]
    yr = bf(yr + (v["b_out"].double()[group] if biases else 0))
    y = plain.combine(yr, places, gates, v["residual"] if residual else None, d)
    dyr, dg = plain.combine_backward(v["dy"], yr, places, gates, torch.zeros(n, d))
    dyr = bf(dyr)
    dw_out, _, db_out, _ = plain.weights_gradient(dyr, h, at)
    dpre = bf(plain.input_gradient(dyr, v["w_out"], at)[0] * plain.slope(bf(pre), act))
    dw_in, _, db_in, _ = plain.weights_gradient(dpre, xr, at)
    dx = plain.combine(bf(plain.input_gradient(dpre, v["w_in"], at)[0]), places, None, None, d)
    # the router's gradient: gates and balance loss
    z = torch.where(part[:, None], v["logits"].double(), 0.0).requires_grad_()
    p = torch.softmax(z, 1)
    g = torch.gather(p, 1, ids)
    if normalize:
        g = g / g.sum(1, keepdim=True)
    tokens = max(1, int(part.sum()))
    f = torch.bincount(ids[part].reshape(-1), minlength=E).double() / (tokens * k)
    loss = E * (f * (p * part[:, None]).sum(0) / tokens).sum()
    ((g * dg * part[:, None]).sum() + loss * v["d_loss"].double()).sum().backward()
    return dict(y=y, loss=loss.detach().view(1), dx=dx, d_logits=z.grad * part[:, None], d_w_in=dw_in, d_w_out=dw_out, d_b_in=db_in, d_b_out=db_out)


def run(layer, v, biases=True, residual=True, **kw):
    c = {n: None if t is None else t.cuda() for n, t in v.items()}
    y, loss = layer.forward(c["x"], c["logits"], c["w_in"], c["w_out"], c["b_in"] if biases else None, c["b_out"] if biases else None, mask=c["mask"],
                            residual=c["residual"] if residual else None)
    got = layer.backward(c["dy"], c["logits"], c["w_in"], c["w_out"], d_loss=c["d_loss"], mask=c["mask"], biases=biases, **kw)
    return dict(got, y=y, loss=loss.clone())


def close(got, want, what):
    got, want = got.cpu().double(), want.double()
    assert got.shape == want.shape and got.isfinite().all(), what
    if want.numel():
        off, top = (got - want).abs().max(), want.abs().max()
        assert off <= 2.0 ** -7 * top + 1e-30, f"{what}: {float(off)} of {float(top)}"
        assert (got - want).norm() <= 2.0 ** -8 * want.norm() + 1e-30, what


@pytest.mark.parametrize("T,E,d,F,k,act,normalize,biases,residual,dtype", [
    (1, 4, 64, 128, 2, "gelu", True, True, True, F32), (37, 8, 72, 136, 2, "gelu", True, True, False, F32), (64, 3, 128, 64, 1, "relu", False, True, True, BF),
    (130, 16, 64, 200, 3, "silu", True, False, True, F32), (300, 5, 256, 264, 1, "none", False, True, False, BF), (5, 200, 8, 8, 8, "gelu", False, False, False, F32)])
def test_against_the_definitions(T, E, d, F, k, act, normalize, biases, residual, dtype):
    v = make(T, E, d, F, k, seed=T)
    layer = MoELayer(E, d, F, T + 5, top_k=k, normalize=normalize, activation=act)
    got = run(layer, v, biases, residual, weights_dtype=dtype)
    want = reference(v, E, d, F, k, act, normalize, biases, residual)
    for name in ("y", "loss", "dx", "d_logits", "d_w_in", "d_w_out") + (("d_b_in", "d_b_out") if biases else ()):
        close(got[name], want[name], name)
    if not residual:
        part = chosen(v, k, normalize)[2]
        assert not got["y"].cpu()[~part].any() and not got["dx"].cpu()[~part].any() and not got["d_logits"].cpu()[~part].any()


def test_a_step_along_the_gradient():
    """The layer's own outputs, moved along each gradient, change as the gradient says: differences of sum(dy y) + d_loss loss in 64 bits of outputs in bf16 are
    off by their rounding, 2^-8 of each |dy y| at most and mostly of either sign, so the step is long enough for its change to be far above that."""
    T, E, d, F, k = 256, 4, 64, 128, 2
    v = make(T, E, d, F, k, seed=9, masked=False)
    layer = MoELayer(E, d, F, T, top_k=k, normalize=True)
    grad = run(layer, v, residual=False)

    def value(u):
        out = run(layer, u, residual=False)
        return float((out["y"].cpu().double() * u["dy"].double()).sum() + 0.5 * out["loss"].cpu().double())

    for name, of in (("d_w_in", "w_in"), ("d_w_out", "w_out"), ("d_b_in", "b_in"), ("d_b_out", "b_out"), ("dx", "x")):
        way = grad[name].cpu().double()
        step = 0.05 * float(v[of].double().norm()) / float(way.norm())
        ends, moved = [], []
        for sign in (1, -1):
            u = dict(v)
            u[of] = (v[of].double() + sign * step * way).to(v[of].dtype)
            ends.append(value(u))
            moved.append(u[of].double())
        want = float((way * (moved[0] - moved[1])).sum())
        noise = 2.0 ** -8 * math.sqrt(2 * float((v["dy"].double() ** 2).sum()) * 2)       # two sums of independent roundings of values of about 1
        curve = 0.05 * abs(want)                                                         # third order of a step of a twentieth, and the roundings within
        assert abs(ends[0] - ends[1] - want) <= 4 * noise + curve, (name, ends, want)


def test_no_tokens_and_nobody():
    layer = MoELayer(4, 64, 64, 16)
    v = make(0, 4, 64, 64, 1, masked=False)
    got = run(layer, v)
    assert got["y"].shape == (0, 64) and got["loss"] == 0 and not got["d_w_in"].any() and not got["d_b_out"].any()
    v = make(7, 4, 64, 64, 1, masked=False)
    v["mask"] = torch.zeros(7, dtype=torch.bool)
    v["x"][:] = float("nan")
    got = run(layer, v)
    assert torch.equal(got["y"].cpu(), v["residual"]) and got["loss"] == 0
    assert not any(got[n].any() for n in ("dx", "d_logits", "d_w_in", "d_w_out", "d_b_in", "d_b_out"))


def test_on_a_stream_of_its_own():
    T, E, d, F, k = 500, 8, 128, 256, 2
    v = make(T, E, d, F, k, seed=4)
    want = run(MoELayer(E, d, F, T, top_k=k), v)
    layer = MoELayer(E, d, F, T, top_k=k, stream=torch.cuda.Stream())
    for i in range(3):
        c = torch.randn(2048, 2048, device="cuda")
        for _ in range(10):
            c = c @ c * 1e-3                                           # work in front of the inputs
        got = run(layer, v)
        junk = [torch.full((T, d), float("nan"), device="cuda", dtype=BF) for _ in range(4)]
        assert all(torch.equal(got[n], want[n]) for n in want), i
        del junk


def test_captured_and_replayed():
    T, E, d, F, k = 700, 8, 128, 256, 2
    v = make(T, E, d, F, k, seed=5)
    c = {n: t.cuda() for n, t in v.items()}
    layer = MoELayer(E, d, F, T, top_k=k, normalize=True)
    args = c["w_in"], c["w_out"]

    def go():
        y, loss = layer.forward(c["x"], c["logits"], *args, c["b_in"], c["b_out"], mask=c["mask"], residual=c["residual"])
        return dict(layer.backward(c["dy"], c["logits"], *args, d_loss=c["d_loss"], mask=c["mask"]), y=y)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    captured = torch.cuda.Stream()
    mine = MoELayer(E, d, F, T, top_k=k, normalize=True, stream=captured)
    eager, layer = layer, mine
    with torch.cuda.graph(graph, stream=captured):
        out = go()
    layer = eager
    for i in range(4):
        c["x"].mul_(0.9), c["logits"].neg_(), c["w_in"].mul_(1.1)
        for t in out.values():
            t.fill_(9)
        graph.replay()
        torch.cuda.synchronize()
        got = {n: t.clone() for n, t in out.items()}
        want = go()
        torch.cuda.synchronize()
        assert all(torch.equal(got[n], want[n]) for n in want), i


def test_refusals():
    with pytest.raises(ValueError):
        MoELayer(4, 64, 64, 16, activation="tanh")
    layer = MoELayer(4, 64, 64, 16)
    v = {n: None if t is None else t.cuda() for n, t in make(7, 4, 64, 64, 1, masked=False).items()}
    ok = (v["x"], v["logits"], v["w_in"], v["w_out"])
    with pytest.raises(RuntimeError):
        layer.backward(v["dy"], v["logits"], v["w_in"], v["w_out"])
    for i, bad in ((0, v["x"].float()), (0, v["x"][:, :32]), (1, v["logits"][:3]), (2, v["w_in"].float()), (2, v["w_in"][:2]), (3, v["w_out"].cpu())):
        args = list(ok)
        args[i] = bad
        with pytest.raises(ValueError):
            layer.forward(*args)
    with pytest.raises(ValueError):
        layer.forward(*ok, v["b_in"].to(BF))
    with pytest.raises(ValueError):
        layer.forward(*ok, residual=v["residual"].float())
    layer.forward(*ok)
    for bad in (v["dy"].float(), v["dy"][:3]):
        with pytest.raises(ValueError):
            layer.backward(bad, *ok[1:])
    assert set(ACTIVATIONS.values()) == {sm.ACT_NONE, sm.ACT_RELU, sm.ACT_GELU, sm.ACT_SILU}
