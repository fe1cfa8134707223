"""Sizes that do not fit the C calls' 32-bit arguments are refused by the binding; cut to 32 bits they would be a smaller call's.  Stand-ins for tensors
whose memory nobody follows: no GPU is needed."""
import pytest
import torch

import paper_2310_18859_amd as sm

MORE = 1 << 32                                                     # 0 in 32 bits


class Tensor:
    """What the binding asks a tensor on the GPU."""
    is_cuda = True

    def __init__(self, shape, dtype):
        self.shape, self.dtype = shape, dtype

    def stride(self):
        return (self.shape[1], 1)

    def numel(self):
        n = 1
        for s in self.shape:
            n *= s
        return n

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 1 << 20


def uint8(n=1 << 50):
    return Tensor((n,), torch.uint8)


def x(rows, cols, dtype=torch.bfloat16):
    return Tensor((rows, cols), dtype)


def ints(*shape):
    return Tensor(shape, torch.int32)


def floats(*shape):
    return Tensor(shape, torch.float32)


@pytest.mark.parametrize("M", [MORE, 3 * MORE, 1 << 31])
@pytest.mark.parametrize("x4", [False, True])
def test_rows_of_a_product(M, x4):
    with pytest.raises((ValueError, sm.SidaError)):
        sm.mx_gemm(x(M, 16, torch.uint8) if x4 else x(M, 32), uint8() if x4 else None, uint8(), uint8(), None, x(M, 8), 0)


def test_columns_of_a_product():
    with pytest.raises((ValueError, sm.SidaError)):
        sm.mx_gemm(x(0, MORE + 32), None, uint8(), uint8(), None, x(0, 8), 0)
    with pytest.raises((ValueError, sm.SidaError)):
        sm.mx_gemm(x(0, 32), None, uint8(), uint8(), None, x(0, MORE + 8), 0)
    with pytest.raises((ValueError, sm.SidaError)):
        sm.mx_gemm(x(0, 32), None, uint8(), uint8(), ints(MORE + 2), x(0, 8), 0)


def test_columns_to_round():
    with pytest.raises((ValueError, sm.SidaError)):
        sm.mx_quantize(x(0, MORE + 32), uint8(), uint8(), 0)


@pytest.mark.parametrize("T,E,k", [(MORE, 8, 2), (0, MORE + 8, 2), (0, 8, MORE + 2)])
def test_router(T, E, k):
    with pytest.raises((ValueError, sm.SidaError)):
        sm.route_backward(x(T, E), ints(T, k), ints(E), x(T, E), 0, d_gates=floats(T, k))
    with pytest.raises((ValueError, sm.SidaError)):
        sm.route(x(T, E), ints(T, k), floats(T, k), ints(E), floats(1), ints(1), 0)   # the workspace's type is wrong: nothing would be launched
    with pytest.raises(ValueError, match="2\\^31"):
        sm.route(x(T, E), ints(T, k), floats(T, k), ints(E), floats(1), uint8(), 0)


def test_sizes():
    """As the library: 0 for what it would not take."""
    for layout in (sm.MX_ROWS, sm.MX_TILES):
        assert sm.mx_codes_bytes(1, MORE + 32, layout) == 0 and sm.mx_scales_bytes(1, MORE + 32, layout) == 0
        assert sm.mx_codes_bytes(MORE, 32, layout) == (16 if layout == sm.MX_ROWS else 32) * MORE and sm.mx_scales_bytes(MORE, 32, layout) == 8 * MORE
    assert sm.mx_codes_bytes(1, 32, MORE) == 0 and sm.mx_codes_bytes(1 << 64, 32, 0) == 0 and sm.mx_scales_bytes(-(1 << 64), 32, 0) == 0
    cfg = sm.SidaRouteConfig(8, 2, sm.FP32, 0)
    assert sm.route_workspace_bytes(cfg, MORE) == 0 and sm.route_workspace_bytes(cfg, MORE + 5) == 0
