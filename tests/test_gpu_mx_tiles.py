"""The grouped product at sizes that reach each of its kernels (which one a size reaches is checked on the host, tests/test_mx_rule_host.py): the sum
split over a workgroup, and tiles of 32 x 128, 64 x 256 and 128 x 256.  Sums are exact in fp32 as in test_gpu_mx.py, and results
the oracle's bits."""
import numpy as np
import pytest
import torch

import paper_2310_18859_amd as sm
from oracle import mx
from test_gpu_mx import DEV, SENTINEL, Experts, bounds, check, dev, product, stream, tokens

pytestmark = pytest.mark.gpu


class Size:
    """counts: tokens of the groups.  The tiles' last ones have 1 to 128 rows, so that each number of 32-row blocks occurs."""

    def __init__(self, kernel, x4, N, K, counts):
        self.kernel, self.x4, self.N, self.K, self.counts = kernel, x4, N, K, counts

    def __repr__(self):
        return f"{self.kernel}-{'x4' if self.x4 else 'bf16'}-{self.N}x{self.K}"

    @property
    def M(self):
        return sum(self.counts)

    def experts(self, seed=1):
        return Experts(len(self.counts), self.N, self.K, seed)


# The ways that results leave: N or N and the rows' distance of 16 bytes, 4 bytes, an odd number of values.  K: whole stages (64 values
# in bf16, 256 in 4 bits) and turns of the loop (four stages in bf16), one stage less, a part of the last one, a single one.
FEW = [300, 1, 0, 131, 64, 33, 97, 15]
MANY = [520, 1, 0, 33, 1600, 64, 65, 1950]
TALL = [20, 0, 178, 346, 640, 1500, 97, 128]
SIZES = (
    [Size("split", x4, 97, 2080, [3, 0, 1, 33]) for x4 in (False, True)]
    + [Size("rows32", x4, N, K, FEW) for x4 in (False, True) for N, K in ((136, 32), (97, 96), (130, 256), (257, 288), (520, 384), (131, 416), (256, 544))]
    + [Size("rows64", False, N, K, MANY) for N, K in ((1600, 32), (1537, 64), (1538, 96), (1792, 256), (1537, 288), (1928, 384), (1666, 416), (1552, 544))]
    + [Size("rows64", True, N, K, MANY) for N, K in ((1600, 32), (1537, 96), (1538, 256), (1792, 288), (1667, 544), (1928, 1024))]
    + [Size("rows128", True, N, K, TALL) for N, K in ((1537, 2080), (1794, 2048), (1800, 2336))]
)


@pytest.mark.parametrize("y_type", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("size", SIZES, ids=repr)
def test_sizes(size, y_type):
    check(size.experts(size.N + size.K), size.M, bounds(size.counts), size.x4, y_type, relu=size.K % 64 == 0, pad_x=0 if size.x4 else 8)


ALIGNED = (
    [Size("split", x4, N, 1024, [3, 40]) for x4 in (False, True) for N in (96, 97, 98)]
    + [Size("rows32", x4, N, 160, FEW) for x4 in (False, True) for N in (128, 129, 130)]
    + [Size("rows64", x4, N, 160, MANY) for x4 in (False, True) for N in (1664, 1665, 1666)]
    + [Size("rows128", True, N, 2048, TALL) for N in (1664, 1665, 1666)]
)


@pytest.mark.parametrize("pad_y,shift_y", [(0, 1), (8, 0), (2, 0), (3, 0), (7, 3)])
@pytest.mark.parametrize("size", ALIGNED, ids=repr)
def test_results_at_any_alignment(size, pad_y, shift_y):
    """Nothing in front of, between and behind the rows of results is written."""
    ex = experts_of(size)
    for y_type in (torch.bfloat16, torch.float32):
        check(ex, size.M, bounds(size.counts), size.x4, y_type, pad_y=pad_y, shift_y=shift_y)


_MADE = {}


def experts_of(size):
    """The last size's experts, made once."""
    if repr(size) not in _MADE:
        _MADE.clear()
        _MADE[repr(size)] = size.experts()
    return _MADE[repr(size)]


EACH = [Size("split", False, 100, 1056, [20, 13]), Size("split", True, 100, 1056, [20, 13]), Size("rows32", False, 260, 160, FEW),
        Size("rows32", True, 260, 160, FEW), Size("rows64", False, 1540, 160, MANY), Size("rows64", True, 1540, 160, MANY), Size("rows128", True, 1540, 2080, TALL)]


@pytest.mark.parametrize("relu", [False, True])
@pytest.mark.parametrize("size", EACH, ids=repr)
def test_what_is_no_number_stays_where_it_is(size, relu):
    """NaN and infinities of an expert's block reach one column of its own rows, a token's its own row; rows of no group and what lies behind
    a row's values reach nobody."""
    ex = size.experts(3)
    ex.scales[0, 70, -1] = 255
    ex.upload()
    at, behind = 7, 5
    offsets = at + bounds(size.counts)
    M = int(offsets[-1]) + behind
    x, xd, xs = tokens(M, size.K, size.x4, 4)
    rows = [at, int(offsets[1]) - 1, int(offsets[-1]) - 1]              # a NaN each, in the first, last or middle block
    outside = np.r_[0:at, M - behind:M]
    if size.x4:
        blocks = size.K // 32
        for r, b in zip(rows, (0, blocks - 1, blocks // 2)):
            xs.view(M, -1)[r, b] = 255
            x[r, b * 32:b * 32 + 32] = np.nan
        xs.view(M, -1)[torch.from_numpy(outside).to(DEV)] = 255
        xd_in = xd
    else:
        for r, c in zip(rows, (0, size.K - 1, size.K // 2)):
            xd[r, c], x[r, c] = float("nan"), np.nan
        xd[torch.from_numpy(outside).to(DEV)] = float("inf")
        wide = torch.full((M, size.K + 8), float("nan"), dtype=torch.bfloat16, device=DEV)
        wide[:, :size.K] = xd
        xd_in = wide[:, :size.K]
    y = torch.full((M, size.N), SENTINEL, device=DEV)
    sm.mx_gemm(xd_in, xs, ex.dev_codes, ex.dev_scales, dev(offsets.astype(np.int32)), y, stream(), relu=relu)
    want = product(ex, x, offsets, relu)
    want[outside] = SENTINEL
    nan = np.zeros_like(want, bool)
    nan[rows] = True
    nan[at:int(offsets[1]), 70] = True
    assert np.array_equal(np.isnan(want), nan)
    assert np.array_equal(y.double().cpu().numpy(), want, equal_nan=True)


@pytest.mark.parametrize("byte", [0, 1, 2, 252])
@pytest.mark.parametrize("size", EACH, ids=repr)
def test_first_and_last_powers(size, byte):
    """Experts' powers of two at both ends of what rounding to MXFP4 gives: weights below the smallest normal bf16, and up to 6 * 2^125.  A token
    has one value that is not 0, so that every result is one product: exact, or infinite where fp32 has no such number."""
    ex = size.experts(5)
    ex.scales[:] = byte
    ex.upload()
    g = np.random.default_rng(byte)
    M = size.M
    at = g.integers(0, size.K, M)
    e = g.integers(-20, 100, M) if byte < 3 else g.integers(-126, 3, M)
    if size.x4:
        codes = np.zeros((M, size.K), np.uint8)
        codes[np.arange(M), at] = g.integers(1, 16, M)
        scales = np.repeat((e + 127).astype(np.uint8)[:, None], size.K // 32, 1)
        x = mx.values(codes, scales)
        xd, xs = (dev(v) for v in mx.pack_rows(codes, scales))
    else:
        x = np.zeros((M, size.K))
        x[np.arange(M), at] = np.ldexp(g.choice([-1.5, -1.0, 1.0, 1.75], M), e)
        xd, xs = dev(x, torch.bfloat16), None
    offsets = bounds(size.counts)
    y = torch.empty((M, size.N), device=DEV)
    sm.mx_gemm(xd, xs, ex.dev_codes, ex.dev_scales, dev(offsets.astype(np.int32)), y, stream())
    with np.errstate(over="ignore"):
        want = product(ex, x, offsets).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), want)


@pytest.mark.parametrize("byte", [253, 254])
@pytest.mark.parametrize("size", EACH, ids=repr)
def test_powers_beyond(size, byte):
    """Powers of two that only other programs' codes have.  Weights of 2^128 and more: infinite against bf16 tokens, exact against codes."""
    ex = size.experts(7)
    ex.codes[:, ::2] &= 0xB                                            # every other column of results has small codes only
    ex.scales[:] = byte
    ex.upload()
    if not size.x4:
        assert all((np.abs(w[1::2]) >= 2.0 ** 128).any() for w in ex.w)
        ex.w = [np.where(np.abs(w) >= 2.0 ** 128, np.copysign(np.inf, w), w) for w in ex.w]
    g = np.random.default_rng(byte)
    M = size.M
    at, e = g.integers(0, size.K, M), g.integers(-126, -3, M)
    if size.x4:
        codes = np.zeros((M, size.K), np.uint8)
        codes[np.arange(M), at] = g.integers(1, 16, M)
        scales = np.repeat((e + 127).astype(np.uint8)[:, None], size.K // 32, 1)
        x = mx.values(codes, scales)
        xd, xs = (dev(v) for v in mx.pack_rows(codes, scales))
    else:
        x = np.zeros((M, size.K))
        x[np.arange(M), at] = np.ldexp(g.choice([-1.5, -1.0, 1.0, 1.75], M), e)
        xd, xs = dev(x, torch.bfloat16), None
    offsets = bounds(size.counts)
    y = torch.empty((M, size.N), device=DEV)
    sm.mx_gemm(xd, xs, ex.dev_codes, ex.dev_scales, dev(offsets.astype(np.int32)), y, stream())
    with np.errstate(over="ignore", invalid="ignore"):
        want = product(ex, x, offsets).astype(np.float32)
    assert np.array_equal(y.cpu().numpy(), want, equal_nan=True)


# Weights N(0, 0.02) and tokens N(0, 1), rounded by the library.  An fp32 sum of K products is off by at most K 2^-23 times the sum of their
# magnitudes (each addition rounds, or cuts, a partial sum of at most that size).
@pytest.mark.parametrize("size", EACH, ids=repr)
def test_ordinary_values(size):
    g = torch.Generator(device=DEV).manual_seed(size.N)
    E, N, K, M = len(size.counts), size.N, size.K, size.M
    n = -(-N // 32) * 32                                               # every expert's rows from a stripe of its own on
    w = torch.zeros((E, n, K), device=DEV)
    w[:, :N] = torch.randn((E, N, K), generator=g, device=DEV) * 0.02
    x = torch.randn((M, K), generator=g, device=DEV).bfloat16()
    codes = torch.empty(E * sm.mx_codes_bytes(N, K, sm.MX_TILES), dtype=torch.uint8, device=DEV)
    scales = torch.empty(E * sm.mx_scales_bytes(N, K, sm.MX_TILES), dtype=torch.uint8, device=DEV)
    wv = torch.empty((E, n, K), dtype=torch.bfloat16, device=DEV)
    sm.mx_quantize(w.view(-1, K), codes, scales, stream(), layout=sm.MX_TILES, values=wv)
    xv, xin, xs = x, x, None
    if size.x4:
        xin = torch.empty((M, K // 2), dtype=torch.uint8, device=DEV)
        xs = torch.empty((M, -(-K // 256) * 8), dtype=torch.uint8, device=DEV)
        xv = torch.empty_like(x)
        sm.mx_quantize(x, xin, xs, stream(), values=xv)
    offsets = bounds(size.counts)
    y = torch.empty((M, N), device=DEV)
    sm.mx_gemm(xin, xs, codes, scales, dev(offsets.astype(np.int32)), y, stream())
    got, a, b = y.double().cpu(), xv.double().cpu(), wv.double().cpu()[:, :N]
    for e in range(E):
        r = slice(int(offsets[e]), int(offsets[e + 1]))
        assert bool(((got[r] - a[r] @ b[e].T).abs() <= K * 2.0 ** -23 * (a[r].abs() @ b[e].abs().T)).all()), e


# Rows 32 MiB apart: the last ones more than 2^31 bytes behind the first.
FAR = [Size("rows32", False, 400, 64, [70, 61]), Size("rows64", False, 40960, 32, [70, 61])]


@pytest.mark.parametrize("size", FAR, ids=repr)
def test_far_rows(size):
    ld = (1 << 24) - 8
    ex = size.experts(2)
    x, xd, _ = tokens(size.M, size.K, False, 4)
    far = torch.empty(size.M * ld, dtype=torch.bfloat16, device=DEV).view(size.M, ld)
    far[:, :size.K] = xd
    out = torch.empty(size.M * ld, dtype=torch.bfloat16, device=DEV).view(size.M, ld)
    offsets = bounds(size.counts)
    sm.mx_gemm(far[:, :size.K], None, ex.dev_codes, ex.dev_scales, dev(offsets.astype(np.int32)), out[:, :size.N], stream())
    want = torch.from_numpy(product(ex, x, offsets)).to(torch.bfloat16)
    assert torch.equal(out[:, :size.N].cpu(), want)


@pytest.mark.parametrize("size", EACH, ids=repr)
def test_offsets_outside_and_in_a_graph(size):
    """Groups that begin before the first row and end behind the last one; the call captured on a stream of its own and replayed on other offsets
    and tokens with eager work in between."""
    ex = size.experts(6)
    M = size.M
    off = dev(np.zeros(len(size.counts) + 1, np.int32))
    _, xd, xs = tokens(M, size.K, size.x4, 1)
    y = torch.empty((M, size.N), device=DEV)
    side = torch.cuda.Stream()

    def call(s):
        sm.mx_gemm(xd, xs, ex.dev_codes, ex.dev_scales, off, y, s)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        call(side)
    for i in range(3):
        o = bounds(size.counts)
        if i:
            o[0], o[-1] = -(10 ** i), 10 ** 9
        if i == 2:
            o[1:-1] = np.sort(np.random.default_rng(i).integers(0, M + 1, len(o) - 2))
        x, new, new_s = tokens(M, size.K, size.x4, 10 + i)
        xd.copy_(new)
        if size.x4:
            xs.copy_(new_s)
        off.copy_(dev(o.astype(np.int32)))
        y.fill_(SENTINEL)
        graph.replay()
        torch.cuda.synchronize()
        first = y.clone()
        y.fill_(SENTINEL)
        call(stream())
        assert torch.equal(first, y)
        assert np.array_equal(y.double().cpu().numpy(), product(ex, x, o))
