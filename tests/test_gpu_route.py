"""The router on the GPU against the 64-bit oracle: choice, gates, counts, balance loss and the logits' gradient.

Ids and counts have one right answer.  Gates: exp(v - m) is taken as a power of two of a product rounded once, off by
|v - m| 2^-23 of itself at most (twice the rounding of a number of that size times log2 e), the hardware power and the
division by a sum add a few units in the last place each, the sum of at most 256 terms eight additions deep: below
(|v - m| + 20) 2^-23 of the gate, and (40 + 20) 2^-23 = 7.2e-6 for the logits used here, whose spread is below 40.  Powers below the smallest
normal number are 0.  The loss and gradients are sums of products of these; tolerances stand at the tests."""
import math

import numpy as np
import pytest
import torch

import paper_2310_18859_amd as sm
from oracle import route as ref

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
GATE = 60 * 2.0 ** -23


def stream():
    return torch.cuda.current_stream()


def draw(T, E, dtype, seed, ties=False):
    g = np.random.default_rng(seed)
    z = g.standard_normal((T, E)) * 2 + g.standard_normal((1, E))
    if ties:
        z = np.round(z)
    return torch.from_numpy(z).to(dtype)


def forward(logits, k, mask=None, normalize=False, workspace=None):
    T, E = logits.shape
    cfg = sm.SidaRouteConfig(E, k, sm.BF16 if logits.dtype == torch.bfloat16 else sm.FP32, int(normalize))
    out = {"ids": torch.full((T + 1, k), -7, dtype=torch.int32, device=DEV), "gates": torch.full((T + 1, k), -7.0, device=DEV),
           "counts": torch.full((E + 1,), -7, dtype=torch.int32, device=DEV), "loss": torch.full((2,), -7.0, device=DEV)}
    n = sm.route_workspace_bytes(cfg, T)
    ws = torch.full((n + 64,), 0xFF, dtype=torch.uint8, device=DEV)          # what it holds before does not matter
    sm.route(logits, out["ids"][:T], out["gates"][:T], out["counts"][:E], out["loss"][:1], ws[:n], stream(), mask=mask, normalize=normalize)
    assert (out["ids"][T] == -7).all() and (out["gates"][T] == -7).all() and out["counts"][E] == -7 and out["loss"][1] == -7
    assert (ws[n:] == 0xFF).all()
    return out["ids"][:T].cpu().numpy(), out["gates"][:T].double().cpu().numpy(), out["counts"][:E].cpu().numpy(), float(out["loss"][0])


def check(logits_cpu, k, mask=None, normalize=False, view=None):
    z = logits_cpu.double().numpy()
    ids, gates, counts, loss = ref.forward(z, k, mask, normalize)
    d = (view or (lambda t: t.to(DEV)))(logits_cpu)
    m = None if mask is None else torch.tensor(np.asarray(mask), dtype=torch.uint8, device=DEV)
    got = forward(d, k, m, normalize)
    assert np.array_equal(got[0], ids)
    assert np.array_equal(got[2], counts)
    tol = GATE * (2 if normalize else 1)
    assert np.array_equal(np.isnan(got[1]), np.isnan(gates))
    assert (np.abs(got[1] - gates) <= tol * np.abs(gates) + 2e-38)[~np.isnan(gates)].all()
    # positive terms: off by what p is, and by a sum of T of them in fp32, here at most 2^12 deep
    assert math.isnan(got[3]) if math.isnan(loss) else abs(got[3] - loss) <= (GATE + 2 ** 12 * 2.0 ** -24) * loss
    return d, m, ids, counts


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,k,normalize", [(1, 1, 1, False), (1, 8, 8, True), (3, 7, 2, False), (64, 128, 1, False), (65, 64, 2, True), (200, 129, 3, True),
                                             (255, 256, 8, False), (256, 16, 1, False), (257, 256, 1, True), (700, 31, 1, False), (1111, 64, 2, True),
                                             (4000, 20, 3, False)])
def test_forward(T, E, k, normalize, dtype):
    g = np.random.default_rng(T)
    check(draw(T, E, dtype, T * 7 + E), k, None, normalize)
    check(draw(T, E, dtype, T * 7 + E + 1, ties=True), k, (g.random(T) < 0.8), normalize)


def test_many_rows():
    """More rows than one round of every workgroup takes; a sample of tokens against the oracle, the sums against torch in 64 bits."""
    T, E, k = 40000, 96, 2
    z = draw(T, E, torch.float32, 3)
    got = forward(z.to(DEV), k)
    p = torch.softmax(z.double(), 1)
    at = np.random.default_rng(1).integers(0, T, 200)
    ids, gates, _, _ = ref.forward(z.double().numpy()[at], k)
    assert np.array_equal(got[0][at], ids) and (np.abs(got[1][at] - gates) <= GATE * gates).all()
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :k]
    counts = torch.bincount(order.reshape(-1), minlength=E)
    assert np.array_equal(got[2], counts.numpy())
    loss = float(E * (counts.double() / (T * k) * p.mean(0)).sum())
    assert abs(got[3] - loss) <= (GATE + 2 ** 12 * 2.0 ** -24) * loss


def test_same_bits_again():
    z = draw(5000, 128, torch.bfloat16, 8).to(DEV)
    a, b = forward(z, 2), forward(z, 2)
    assert all(np.array_equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("k", [1, 2, 4])
@pytest.mark.parametrize("normalize", [False, True])
def test_infinities_and_nan(k, normalize):
    """Experts shut off by -infinity, rows of nothing else, a +infinity, NaN in rows that take part and in masked ones."""
    inf, nan = math.inf, math.nan
    z = torch.tensor([[0.0, -inf, 1.0, -inf], [-inf] * 4, [-inf, -inf, -inf, 2.0], [nan] * 4, [1.0, nan, inf, 0.0], [-1e30, -1e30, -2e30, -inf],
                      [-3.4e38, -3.4e38, -3.4e38, -3.4e38], [3.4e38, -3.4e38, 1.0, 0.0], [0.0, -0.0, 0.0, -0.0]])
    clean = [1, 1, 1, 0, 0, 1, 1, 1, 1]
    for dtype in (torch.float32, torch.bfloat16):
        d, m, ids, counts = check(z.to(dtype), k, clean, normalize)
        grad = torch.full((9, 4), 5.0, dtype=dtype, device=DEV)
        dg = np.random.default_rng(k).standard_normal((9, k))
        sm.route_backward(d, torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(counts.astype(np.int32)).to(DEV), grad, stream(),
                          d_gates=torch.tensor(dg, dtype=torch.float32, device=DEV), mask=m, normalize=normalize)
        want = ref.backward(d.double().cpu().numpy(), ids, counts, dg.astype(np.float32).astype(np.float64), 0.0, clean, normalize)
        got = grad.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), np.isnan(want))              # 3.4e38 is an infinity in bf16
        assert (got[[1, 3, 4]] == 0).all()
        fine = ~np.isnan(want)
        assert np.abs(got - want)[fine].max() <= (2 ** -8 if dtype == torch.bfloat16 else 1e-5) * max(1.0, np.abs(want[fine]).max())
        check(z.to(dtype), k, None, normalize)                            # a NaN that takes part makes gates and loss NaN, ids stay in range


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_nobody_takes_part(dtype):
    z = draw(70, 32, dtype, 1)
    check(z, 2, np.zeros(70))
    check(torch.full((300, 32), -math.inf, dtype=dtype), 2)
    g = torch.full((70, 32), 3.0, dtype=dtype, device=DEV)
    sm.route_backward(z.to(DEV), torch.zeros((70, 2), dtype=torch.int32, device=DEV), torch.zeros(32, dtype=torch.int32, device=DEV), g, stream(),
                      d_gates=torch.ones((70, 2), device=DEV), d_loss=torch.ones(1, device=DEV), mask=torch.zeros(70, dtype=torch.bool, device=DEV))
    assert (g == 0).all()


def test_no_tokens():
    z = torch.empty((0, 16), device=DEV)
    ids, gates, counts, loss = forward(z, 2)
    assert (counts == 0).all() and loss == 0


def views(dtype):
    def shifted(t):
        buf = torch.empty(t.numel() + 1, dtype=dtype, device=DEV)
        buf[1:] = t.reshape(-1).to(DEV)
        return buf[1:].view(t.shape)

    def strided(pad):
        def go(t):
            wide = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=dtype, device=DEV)
            wide[:, :t.shape[1]] = t.to(DEV)
            return wide[:, :t.shape[1]]
        return go

    return [shifted, strided(8), strided(1)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("E", [24, 64, 256])
@pytest.mark.parametrize("which", [0, 1, 2])
def test_strides_and_alignment(E, dtype, which):
    view = views(dtype)[which]
    z = draw(90, E, dtype, E)
    check(z, 2, None, True, view)
    backward(z, 2, None, True, view)


# The gradient p (dp - sum p dp): p is off by GATE of itself, dp by a few units in its last place, the sum over at most
# 256 columns by GATE + 2^-19 of the largest |dp|: below (4 GATE + 2^-18) p max|dp| in all, and one rounding to bf16 on top.
def backward(z, k, mask, normalize, view=None, d_loss=0.3, in_place=False, with_gates=True):
    T, E = z.shape
    zz = z.double().numpy()
    ids, _, counts, _ = ref.forward(zz, k, mask, normalize)
    g = np.random.default_rng(T * E + k)
    dg = g.standard_normal((T, k)).astype(np.float32) if with_gates else None
    want = ref.backward(zz, ids, counts, None if dg is None else dg.astype(np.float64), d_loss or 0.0, mask, normalize)
    d = (view or (lambda t: t.to(DEV)))(z)
    out = d if in_place else (view(torch.zeros_like(z)) if view else torch.empty_like(d))
    sm.route_backward(d, torch.from_numpy(ids.astype(np.int32)).to(DEV), torch.from_numpy(counts.astype(np.int32)).to(DEV), out, stream(),
                      d_gates=None if dg is None else torch.from_numpy(dg).to(DEV),
                      d_loss=None if d_loss is None else torch.tensor([d_loss], device=DEV),
                      mask=None if mask is None else torch.tensor(np.asarray(mask), dtype=torch.bool, device=DEV), normalize=normalize)
    got = out.double().cpu().numpy()
    for t in range(T):
        p = ref.softmax(zz[t])
        n = max(1, counts.sum() / k)
        most = abs(d_loss or 0.0) * E / n * counts.max() / (n * k)
        if dg is not None:
            q = p[ids[t]].sum() if normalize else 1.0
            most += np.abs(dg[t]).sum() * (2 if normalize else 1) / q
        tol = (4 * GATE * (3 if normalize else 1) + 2.0 ** -18) * p * most + 1e-37
        if z.dtype == torch.bfloat16:
            tol = tol * 1.01 + np.abs(want[t]) * 2.0 ** -8
        assert (np.abs(got[t] - want[t]) <= tol).all(), t


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,E,k,normalize", [(1, 1, 1, True), (1, 8, 8, True), (3, 7, 2, False), (64, 128, 1, False), (65, 64, 2, True), (200, 129, 3, True),
                                             (255, 256, 8, False), (257, 256, 1, True), (700, 31, 1, False)])
def test_backward(T, E, k, normalize, dtype):
    g = np.random.default_rng(T)
    backward(draw(T, E, dtype, T + E), k, None, normalize)
    backward(draw(T, E, dtype, T + E + 1), k, (g.random(T) < 0.8), normalize)
    backward(draw(T, E, dtype, T + E + 2), k, None, normalize, d_loss=None)
    backward(draw(T, E, dtype, T + E + 3), k, None, normalize, with_gates=False)
    backward(draw(T, E, dtype, T + E + 4), k, None, normalize, in_place=True)


def test_gradient_against_differences_of_the_kernel():
    """Central differences of the kernel's own gates and loss in fp32: a step of 2^-6 with values of order 1, whose last
    place is 2^-24, gives 2^-17 of noise, and the third derivative 2^-12 / 6 of curvature: 1e-4 in all."""
    T, E, k, h = 4, 12, 2, 2.0 ** -6
    z = draw(T, E, torch.float32, 31)
    g = np.random.default_rng(2)
    dg, dl = g.standard_normal((T, k)).astype(np.float32), 0.5
    ids, _, counts, _ = forward(z.to(DEV), k, normalize=True)
    grad = torch.empty((T, E), device=DEV)
    sm.route_backward(z.to(DEV), torch.from_numpy(ids).to(DEV), torch.from_numpy(counts).to(DEV), grad, stream(),
                      d_gates=torch.from_numpy(dg).to(DEV), d_loss=torch.tensor([dl], device=DEV), normalize=True)
    compared = 0
    for t in range(T):
        for e in range(E):
            v = []
            for s in (h, -h):
                y = z.clone()
                y[t, e] += s
                i, gates, _, loss = forward(y.to(DEV), k, normalize=True)
                if np.array_equal(i, ids):
                    v.append((gates * dg).sum() + dl * loss)
            if len(v) < 2:                                                 # a step that changes the choice has no derivative
                continue
            compared += 1
            assert abs((v[0] - v[1]) / (2 * h) - float(grad[t, e])) < 1e-4
    assert compared >= T * E - 4


def test_ids_outside_add_nothing():
    z = draw(30, 16, torch.float32, 4).to(DEV)
    counts = torch.full((16,), 2, dtype=torch.int32, device=DEV)
    dg, dl = torch.ones((30, 2), device=DEV), torch.ones(1, device=DEV)
    a, b = torch.empty_like(z), torch.empty_like(z)
    bad = torch.tensor([[-1, 16]] * 15 + [[2 ** 31 - 1, -2 ** 31]] * 15, dtype=torch.int32, device=DEV)
    for normalize in (False, True):
        sm.route_backward(z, bad, counts, a, stream(), d_gates=dg, d_loss=dl, normalize=normalize)
        sm.route_backward(z, bad, counts, b, stream(), d_loss=dl, normalize=normalize)
        assert torch.equal(a, b)


def test_on_another_stream_and_in_a_graph():
    T, E, k = 2000, 64, 2
    side = torch.cuda.Stream()
    z = torch.zeros((T, E), device=DEV)
    ids = torch.zeros((T, k), dtype=torch.int32, device=DEV)
    gates, grad = torch.zeros((T, k), device=DEV), torch.zeros((T, E), device=DEV)
    counts, loss = torch.zeros(E, dtype=torch.int32, device=DEV), torch.zeros(1, device=DEV)
    dg, dl = torch.ones((T, k), device=DEV), torch.ones(1, device=DEV)
    ws = torch.zeros(sm.route_workspace_bytes(sm.SidaRouteConfig(E, k, sm.FP32, 0), T), dtype=torch.uint8, device=DEV)

    def both(s):
        sm.route(z, ids, gates, counts, loss, ws, s)
        sm.route_backward(z, ids, counts, grad, s, d_gates=dg, d_loss=dl)

    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        both(side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        both(side)
    for i in range(4):
        z.copy_(draw(T, E, torch.float32, 50 + i))
        graph.replay()
        torch.cuda.synchronize()
        first = [t.clone() for t in (ids, gates, counts, loss, grad)]
        for t in (ids, gates, counts, loss, grad, ws):
            t.zero_()
        both(stream())
        assert all(torch.equal(a, b) for a, b in zip(first, (ids, gates, counts, loss, grad)))
        assert float(counts.sum()) == T * k
