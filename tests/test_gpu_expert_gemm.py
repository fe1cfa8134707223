"""Products of plain bf16 experts with their gradients against the definitions in 64 bits.

Tolerances.  A sum of n products of bf16 values, each exact in fp32, is off by at most (n + 2) roundings of the sum of magnitudes S (any
order, a bias or a residual added): (n + 2) 2^-24 S.  An activation v s(u), s the sigmoid: u takes nine roundings, no cancellation, so exp(-u) is off
by 9 |u| 2^-24 of itself and s by no more; two for each of exp, reciprocal and product: (9 |u| + 8) 2^-24 |v s|, and what v is off by times the
largest slope, 1.2.  The slope s + v (1 - s) s u' adds terms of which each is off by as much, four roundings more: (27 |u| + 24) 2^-24 (s + |v| s (1 - s) u').  Then
half a step of the result's type: 2^-8 of the value in bf16, 2^-24 in fp32.  Beyond u = 88 all of it is 0 or the value itself."""
import math

import pytest
import torch

import paper_2310_18859_amd as sm
from oracle import experts as plain

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}
BF, F32 = torch.bfloat16, torch.float32
ACTS = {"none": sm.ACT_NONE, "relu": sm.ACT_RELU, "gelu": sm.ACT_GELU, "silu": sm.ACT_SILU}
E24 = 2.0 ** -24


def stream():
    return torch.cuda.current_stream()


def strided(t, pad):
    """t on the GPU with `pad` NaN between its rows."""
    base = torch.full((t.shape[0], t.shape[1] + pad), float("nan"), dtype=t.dtype, device="cuda")
    base[:, :t.shape[1]] = t.cuda()
    return base[:, :t.shape[1]]


def buffer(rows, cols, dtype, pad, fill=7.0):
    return strided(torch.full((rows, cols), fill, dtype=dtype), pad)


def bounds_of(sizes, front=0):
    out = [front]
    for n in sizes:
        out.append(out[-1] + n)
    return out


def act_error(v, v_err, act):
    """What the activation of a value that is off by v_err may be off by."""
    if act in ("none", "relu"):
        return v_err
    u = plain.argument(v, act).abs().clamp(max=88)
    return 1.2 * v_err + (9 * u + 8) * E24 * plain.activation(v, act).abs() + 2.0 ** -100


def slope_error(v, act):
    if act in ("none", "relu"):
        return torch.zeros_like(v)
    u = plain.argument(v, act)
    du = 1.0 if act == "silu" else 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v ** 2)
    s = torch.sigmoid(u)
    return (27 * u.abs().clamp(max=88) + 24) * E24 * (s + v.abs() * s * torch.sigmoid(-u) * du) + 2.0 ** -60


def inputs(seed, *shapes):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(s, generator=g) for s in shapes]


# sizes of the groups, N, K: single rows, empty groups, odd sizes, more than a tile, long sums
SHAPES = [([1], 8, 8), ([1], 4096, 1024), ([1, 0, 1], 264, 72), ([3, 0, 0, 5, 1], 72, 264), ([0, 31, 32, 33, 0], 136, 1000), ([65, 1, 129], 520, 328),
          ([300, 0, 7], 256, 512), ([257], 648, 200), ([16] * 40, 64, 128), ([700, 2, 90], 1024, 64), ([0, 0], 64, 64), ([40, 33], 2048, 2056)]


@pytest.mark.parametrize("sizes,N,K", SHAPES)
@pytest.mark.parametrize("act,bias,pre,residual,dtype,pad", [
    ("none", False, False, False, BF, 0), ("none", False, False, False, F32, 8), ("gelu", True, True, False, BF, 0), ("silu", True, True, True, F32, 16),
    ("relu", False, True, True, BF, 8), ("gelu", False, False, True, BF, 0)])
def test_product(sizes, N, K, act, bias, pre, residual, dtype, pad):
    at = bounds_of(sizes, 3)                                        # three rows in front and two behind belong to nobody
    M, groups = at[-1] + 2, len(sizes)
    x, w, b, res = inputs(N + K, (M, K), (groups, N, K), (groups, N), (M, N))
    x, w, res = x.to(BF), (w / math.sqrt(K)).to(BF), res.to(dtype)
    x[:3], x[-2:] = float("nan"), float("inf")
    y, p = buffer(M, N, dtype, pad), buffer(M, N, BF, pad) if pre else None
    sm.expert_gemm(strided(x, pad), w.cuda(), torch.tensor(at, dtype=torch.int32, device="cuda"), y, stream(), bias=b.cuda() if bias else None,
                   activation=ACTS[act], pre=p, residual=strided(res, pad) if residual else None)
    v, size = plain.product(x[at[0]:at[-1]], w, [a - at[0] for a in at])
    group = torch.bucketize(torch.arange(v.shape[0]), torch.tensor(at[1:]) - at[0], right=True)
    if bias and v.numel():
        v, size = v + b.double()[group], size + b.double().abs()[group]
    err = (K + 2) * E24 * size
    for t in (y, p):
        if t is not None:
            assert t[:3].eq(7).all() and t[-2:].eq(7).all()
    inner = slice(at[0], at[-1])
    if pre:
        assert ((p[inner].cpu().double() - v).abs() <= err + HALF[BF] * (v.abs() + err)).all()
    want, tol = plain.activation(v, act), act_error(v, err, act)
    if residual:
        want = want + res[inner].double()
        tol = tol + E24 * (want.abs() + tol)
    assert ((y[inner].cpu().double() - want).abs() <= tol + HALF[dtype] * (want.abs() + tol)).all()


@pytest.mark.parametrize("sizes,N,K", SHAPES)
@pytest.mark.parametrize("act,dtype,pad", [("none", BF, 0), ("none", F32, 8), ("gelu", BF, 0), ("silu", F32, 16), ("relu", BF, 8)])
def test_input_gradient(sizes, N, K, act, dtype, pad):
    at = bounds_of(sizes, 3)
    M, groups = at[-1] + 2, len(sizes)
    dy, w, pre = inputs(N + 2 * K, (M, N), (groups, N, K), (M, K))
    dy, w, pre = dy.to(BF), (w / math.sqrt(N)).to(BF), (pre * 2).to(BF)
    dy[:3], dy[-2:] = float("nan"), float("inf")
    dx = buffer(M, K, dtype, pad)
    given = strided(pre, pad) if act != "none" else None
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    sm.expert_gemm_input(strided(dy, pad), w.cuda(), offsets, dx, stream(), pre=given, activation=ACTS[act])
    inner = slice(at[0], at[-1])
    v, size = plain.input_gradient(dy[inner], w, [a - at[0] for a in at])
    p = pre[inner].double()
    slope, slope_err = plain.slope(p, act), slope_error(p, act)
    err = (N + 2) * E24 * size
    want, tol = v * slope, err * (slope.abs() + slope_err) + v.abs() * slope_err
    assert dx[:3].eq(7).all() and dx[-2:].eq(7).all()
    assert ((dx[inner].cpu().double() - want).abs() <= tol + (HALF[dtype] + E24) * (want.abs() + tol)).all()
    if act != "none" and dtype == BF:                               # in place of the values in front of the activation
        sm.expert_gemm_input(strided(dy, pad), w.cuda(), offsets, given, stream(), pre=given, activation=ACTS[act])
        assert torch.equal(given[inner], dx[inner])


@pytest.mark.parametrize("sizes,N,K", SHAPES + [([5000, 9], 24, 40), ([0, 2500], 264, 136)])
@pytest.mark.parametrize("dtype,bias,pad", [(BF, True, 0), (F32, True, 8), (F32, False, 0)])
def test_weights_gradient(sizes, N, K, dtype, bias, pad):
    at = bounds_of(sizes, 3)
    M, groups = at[-1] + 2, len(sizes)
    dy, x = (t.to(BF) for t in inputs(2 * N + K, (M, N), (M, K)))
    dy[:3], x[-2:] = float("nan"), float("inf")
    dw = torch.full((groups, N, K), 7.0, dtype=dtype, device="cuda")
    db = torch.full((groups, N), 7.0, device="cuda") if bias else None
    ws = torch.empty(max(16, sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(groups, N, K, sm.FP32 if dtype == F32 else sm.BF16, 0), M)),
                     dtype=torch.uint8, device="cuda")
    sm.expert_gemm_weights(strided(dy, pad), strided(x, pad), torch.tensor(at, dtype=torch.int32, device="cuda"), dw, ws, stream(), d_bias=db)
    want, size, want_b, size_b = plain.weights_gradient(dy, x, at)
    n = max(sizes) + 2
    tol = n * E24 * size
    assert ((dw.cpu().double() - want).abs() <= tol + HALF[dtype] * (want.abs() + tol)).all()
    if bias:
        assert ((db.cpu().double() - want_b).abs() <= n * E24 * size_b).all()
    for g, s in enumerate(sizes):
        assert s or not dw[g].any()


def test_one_group_without_offsets():
    x, w, dy = (t.to(BF).cuda() for t in inputs(5, (70, 96), (40, 96), (70, 40)))
    offsets = torch.tensor([0, 70], dtype=torch.int32, device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    got = []
    for o, m in ((None, w), (offsets, w[None])):
        y, dx, dw = torch.empty((70, 40), device="cuda"), torch.empty((70, 96), device="cuda"), torch.empty(m.shape, device="cuda")
        sm.expert_gemm(x, m, o, y, stream())
        sm.expert_gemm_input(dy, m, o, dx, stream())
        sm.expert_gemm_weights(dy, x, o, dw, ws, stream())
        got.append((y, dx, dw.view(40, 96)))
    assert all(torch.equal(a, b) for a, b in zip(*got))


def test_in_place_residual():
    x, w, res = (t.to(BF).cuda() for t in inputs(6, (50, 64), (72, 64), (50, 72)))
    y = torch.empty_like(res)
    sm.expert_gemm(x, w, None, y, stream(), activation=sm.ACT_SILU, residual=res)
    sm.expert_gemm(x, w, None, res, stream(), activation=sm.ACT_SILU, residual=res)
    assert torch.equal(res, y)


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_activations_at_the_ends(act):
    """Products that are +-huge, infinite and NaN: what the activation and its slope make of them."""
    big = torch.tensor([3e38, 1e20, 100.0, 9.5, 0.0, -9.5, -100.0, -1e20, -3e38, float("inf"), -float("inf"), float("nan")]).to(BF)
    n = big.numel()
    x = torch.zeros((n, 8), dtype=BF)
    x[:, 0] = big
    w = torch.zeros((8, 8), dtype=BF)
    w[0, 0] = 1
    y, pre = torch.empty((n, 8), device="cuda"), torch.empty((n, 8), dtype=BF, device="cuda")
    w = w.cuda()
    bias = torch.zeros((1, 8), device="cuda")
    sm.expert_gemm(x[:9].cuda(), w, None, y[:9], stream(), bias=bias, activation=ACTS[act], pre=pre[:9])
    v = big[:9].double()
    assert ((y[:9, 0].cpu().double() - plain.activation(v, act)).abs() <= act_error(v, v * 0, act) + E24 * v.abs()).all()
    assert torch.equal(pre[:9, 0].cpu(), big[:9])
    dy = torch.zeros((n, 8), dtype=BF, device="cuda")
    dy[:, 0] = 1
    pre = x.cuda()
    dx = torch.empty((n, 8), device="cuda")
    sm.expert_gemm_input(dy, w, None, dx, stream(), pre=pre, activation=ACTS[act])
    want = torch.tensor([1.0 if float(b) > 9 else 0.0 for b in big[:11]])
    want[4] = 0.0 if act == "relu" else 0.5
    off = (dx[:11, 0].cpu() - want).abs()
    assert (off <= (2e-3 if act == "silu" else 1e-6)).all(), off       # silu's slope at 9.5: 1 + 9.5 e^-9.5 and less beyond
    assert dx[11, 0].isnan()
    b = torch.zeros((1, 8), device="cuda")
    for value, want in ((float("inf"), float("inf")), (-float("inf"), 0.0), (float("nan"), float("nan"))):
        b[0, 3] = value
        sm.expert_gemm(torch.ones((1, 8), dtype=BF, device="cuda"), w, None, y[:1], stream(), bias=b, activation=ACTS[act])
        assert torch.equal(y[0, 3].cpu().nan_to_num(nan=5.0), torch.tensor(want).nan_to_num(nan=5.0))


def test_infinities_and_nan_stay_in_their_rows_and_groups():
    sizes, N, K = [40, 50], 72, 136
    at = bounds_of(sizes)
    x, w, dy = (t.to(BF) for t in inputs(8, (90, K), (2, N, K), (90, N)))
    x[7, 3], x[60, 5], dy[41] = float("nan"), float("inf"), float("nan")
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    y = torch.empty((90, N), dtype=BF, device="cuda")
    sm.expert_gemm(x.cuda(), w.cuda(), offsets, y, stream())
    bad = torch.zeros(90, dtype=torch.bool)
    bad[7] = bad[60] = True
    assert torch.equal(~y.isfinite().all(1).cpu(), bad) and y[7].isnan().all()
    dw = torch.empty((2, N, K), device="cuda")
    ws = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
    sm.expert_gemm_weights(dy.cuda(), x.cuda(), offsets, dw, ws, stream())
    assert dw[0, :, 3].isnan().all() and dw[0].isnan().sum() == N and dw[1].isnan().all()


def test_offsets_outside_are_clamped():
    x, w = (t.to(BF).cuda() for t in inputs(9, (20, 64), (3, 32, 64)))
    y = torch.full((20, 32), 7.0, device="cuda")
    sm.expert_gemm(x, w, torch.tensor([-5, 6, 6, 99], dtype=torch.int32, device="cuda"), y, stream())
    z = torch.empty_like(y)
    sm.expert_gemm(x, w, torch.tensor([0, 6, 6, 20], dtype=torch.int32, device="cuda"), z, stream())
    assert torch.equal(y, z)
    y.fill_(7.0)
    sm.expert_gemm(x, w, torch.tensor([8, 8, 8, 8], dtype=torch.int32, device="cuda"), y, stream())
    assert y.eq(7).all()


def test_offsets_that_do_not_ascend_stay_inside():
    """Twice as many parts as ascending offsets could make: nothing behind the workspace, the gradients and the rows is written."""
    M, groups, N, K = 16385, 4, 520, 264
    dy, x = (t.to(BF).cuda() for t in inputs(10, (M, N), (M, K)))
    at = torch.tensor([0, M, 0, M, 0], dtype=torch.int32, device="cuda")
    need = sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(groups, N, K, sm.FP32, 0), M)
    assert need
    ws = torch.full((3 * need,), 7, dtype=torch.uint8, device="cuda")
    dw, db = (torch.full((groups + 1,) + shape, 7.0, device="cuda") for shape in ((N, K), (N,)))
    sm.expert_gemm_weights(dy, x, at, dw[:groups], ws[:need], stream(), d_bias=db[:groups])
    assert ws[need:].eq(7).all() and dw[groups].eq(7).all() and db[groups].eq(7).all()
    w = dw[:groups].to(BF)
    y = torch.full((M + 9, N), 7.0, dtype=BF, device="cuda")
    sm.expert_gemm(x, w, at, y[:M], stream())
    assert y[M:].eq(7).all()


def test_long_matrices():
    """Rows whose offsets in bytes and in values pass 32 bits."""
    M, N, K = 1100000, 2048, 64
    x, w = torch.zeros((M, K), dtype=BF, device="cuda"), torch.randn((N, K), device="cuda").to(BF)
    x[-5:] = torch.randn((5, K), device="cuda").to(BF)
    y = torch.empty((M, N), dtype=BF, device="cuda")
    sm.expert_gemm(x, w, None, y, stream())
    few = torch.empty((5, N), dtype=BF, device="cuda")
    sm.expert_gemm(x[-5:], w, None, few, stream())
    v, size = plain.product(x[-5:].cpu(), w[None].cpu(), [0, 5])
    tol = (K + 2) * E24 * size
    for got in (y[-5:], few):
        assert ((got.cpu().double() - v).abs() <= tol + HALF[BF] * (v.abs() + tol)).all()
    assert not y[:-5].any()
    dx = torch.empty((M, K), dtype=BF, device="cuda")
    sm.expert_gemm_input(y, w, None, dx, stream())
    v, size = plain.input_gradient(y[-5:].cpu(), w[None].cpu(), [0, 5])
    tol = (N + 2) * E24 * size
    assert ((dx[-5:].cpu().double() - v).abs() <= tol + HALF[BF] * (v.abs() + tol)).all() and not dx[:-5].any()
    dw, ws = torch.empty((N, K), device="cuda"), torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
    sm.expert_gemm_weights(y, x, None, dw, ws, stream())
    want, size, _, _ = plain.weights_gradient(y[-5:].cpu(), x[-5:].cpu(), [0, 5])
    assert ((dw.cpu().double() - want[0]).abs() <= (M + 2) * E24 * size[0]).all()


def test_repeats_bit_for_bit_and_from_a_graph():
    sizes, N, K = [200, 0, 31, 500], 264, 520
    at = torch.tensor(bounds_of(sizes), dtype=torch.int32, device="cuda")
    M = sum(sizes)
    x, w, dy, b = inputs(11, (M, K), (4, N, K), (M, N), (4, N))
    x, w, dy, b = x.to(BF).cuda(), w.to(BF).cuda(), dy.to(BF).cuda(), b.cuda()
    y, pre, dx, dw, db = (torch.empty(s, dtype=t, device="cuda") for s, t in (((M, N), BF), ((M, N), BF), ((M, K), F32), ((4, N, K), BF), ((4, N), F32)))
    ws = torch.empty(1 << 26, dtype=torch.uint8, device="cuda")

    def go():
        sm.expert_gemm(x, w, at, y, stream(), bias=b, activation=sm.ACT_GELU, pre=pre)
        sm.expert_gemm_input(dy, w, at, dx, stream(), pre=x, activation=sm.ACT_SILU)
        sm.expert_gemm_weights(dy, x, at, dw, ws, stream(), d_bias=db)

    side = torch.cuda.Stream()
    side.wait_stream(stream())
    with torch.cuda.stream(side):
        go()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        go()
    for i in range(4):
        x.mul_(0.5), dy.neg_()
        for t in (y, pre, dx, dw, db):
            t.fill_(3)
        ws.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, pre, dx, dw, db)]
        go()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(got, (y, pre, dx, dw, db)))
