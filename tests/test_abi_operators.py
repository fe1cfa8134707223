"""What the operators without a context refuse, before anything is enqueued: no GPU is needed."""
import ctypes as C

import pytest
import torch

import paper_2310_18859_amd as sm

OK, EINVAL, ENOSPC = 0, -1, -2
P = 1 << 20                                                       # an aligned address that is never followed


def quantize(x=P, x_type=sm.BF16, rows=4, cols=64, ld=64, layout=sm.MX_ROWS, codes=P, scales=P, values=0):
    return sm.lib().sida_mx_quantize(x, x_type, rows, cols, ld, layout, codes, scales, values, 0)


@pytest.mark.parametrize("bad", [dict(x=0), dict(codes=0), dict(scales=0), dict(x=P + 1), dict(x=P + 2, x_type=sm.FP32), dict(codes=P + 8),
                                 dict(scales=P + 4), dict(scales=P + 8, layout=sm.MX_TILES), dict(values=P + 2), dict(x_type=sm.MXFP4), dict(x_type=-1),
                                 dict(rows=-1), dict(cols=0), dict(cols=48), dict(cols=-32), dict(cols=16416, ld=16416), dict(ld=63), dict(ld=1 << 41),
                                 dict(layout=2), dict(rows=1 << 40), dict(rows=1 << 41)])
def test_quantize_refuses(bad):
    assert quantize(**bad) == EINVAL


def test_quantize_of_nothing():
    assert quantize(rows=0, x=0, codes=0, scales=0) == OK


@pytest.mark.parametrize("rows,cols,layout,codes,scales", [(0, 32, 0, 0, 0), (3, 96, 0, 144, 24), (3, 96, 1, 32 * 64, 32 * 8), (33, 288, 1, 64 * 160, 64 * 16),
                                                           (1, 16384, 0, 8192, 512), (-1, 32, 0, 0, 0), (1, 33, 0, 0, 0), (1, 16416, 0, 0, 0), (1, 32, 2, 0, 0)])
def test_sizes(rows, cols, layout, codes, scales):
    assert sm.mx_codes_bytes(rows, cols, layout) == codes and sm.mx_scales_bytes(rows, cols, layout) == scales


def gemm(groups=2, N=64, K=64, x_type=sm.BF16, y_type=sm.BF16, relu=0, x=P, xs=0, ldx=64, M=5, codes=P, scales=P, offsets=P, y=P, ldy=64, cfg=True):
    c = sm.SidaMxGemmConfig(groups, N, K, x_type, y_type, relu)
    return sm.lib().sida_mx_gemm(C.byref(c) if cfg else None, x, xs, ldx, M, codes, scales, offsets, y, ldy, 0)


@pytest.mark.parametrize("bad", [dict(cfg=False), dict(groups=0), dict(groups=257), dict(N=0), dict(N=65537, ldy=65537), dict(K=0), dict(K=40), dict(K=16416, ldx=16416),
                                 dict(x_type=sm.FP32), dict(x_type=3), dict(y_type=sm.MXFP4), dict(x=0), dict(codes=0), dict(scales=0), dict(y=0),
                                 dict(offsets=0), dict(M=-1), dict(M=(1 << 24) + 1), dict(M=1 << 24, N=4096, ldy=4096), dict(ldx=56), dict(ldx=68), dict(ldx=1 << 24), dict(ldy=63),
                                 dict(ldy=1 << 24), dict(x=P + 8), dict(codes=P + 4), dict(scales=P + 2), dict(y=P + 1), dict(y=P + 2, y_type=sm.FP32),
                                 dict(offsets=P + 2), dict(x_type=sm.MXFP4), dict(x_type=sm.MXFP4, xs=P + 4), dict(x_type=sm.MXFP4, xs=P, ldx=72)])
def test_gemm_refuses(bad):
    assert gemm(**bad) == EINVAL


def test_gemm_of_nothing():
    assert gemm(M=0, x=0, y=0, codes=0, scales=0, offsets=0) == OK


def route(E=8, k=2, kind=sm.FP32, logits=P, ld=8, T=5, mask=0, ids=P, gates=P, counts=P, loss=P, ws=P, n=1 << 20, cfg=True):
    c = sm.SidaRouteConfig(E, k, kind, 0)
    return sm.lib().sida_route(C.byref(c) if cfg else None, logits, ld, T, mask, ids, gates, counts, loss, ws, n, 0)


@pytest.mark.parametrize("bad", [dict(cfg=False), dict(E=0), dict(E=257, ld=257), dict(k=0), dict(k=9, E=16, ld=16), dict(k=3, E=2), dict(kind=sm.MXFP4),
                                 dict(logits=0), dict(ids=0), dict(gates=0), dict(counts=0), dict(loss=0), dict(ws=0), dict(ld=7), dict(ld=1 << 24),
                                 dict(T=-1), dict(T=(1 << 26) + 1), dict(logits=P + 2), dict(logits=P + 1, kind=sm.BF16), dict(ids=P + 2), dict(gates=P + 2),
                                 dict(counts=P + 1), dict(loss=P + 2), dict(ws=P + 8)])
def test_route_refuses(bad):
    assert route(**bad) == EINVAL


def test_route_workspace():
    cfg = sm.SidaRouteConfig(64, 2, sm.FP32, 0)
    for T in (0, 1, 256, 257, 100000, 1 << 26):
        n = sm.route_workspace_bytes(cfg, T)
        assert n >= 64 * 8
        assert route(E=64, ld=64, T=T, n=n - 1) == ENOSPC
    assert sm.route_workspace_bytes(cfg, -1) == 0 and sm.route_workspace_bytes(sm.SidaRouteConfig(0, 1, sm.FP32, 0), 5) == 0


def back(E=8, k=2, kind=sm.FP32, logits=P, ld=8, T=5, mask=0, ids=P, counts=P, dg=P, dl=P, out=2 * P, ld_d=8, cfg=True):
    c = sm.SidaRouteConfig(E, k, kind, 0)
    return sm.lib().sida_route_backward(C.byref(c) if cfg else None, logits, ld, T, mask, ids, counts, dg, dl, out, ld_d, 0)


@pytest.mark.parametrize("bad", [dict(cfg=False), dict(E=0), dict(k=9, E=16, ld=16, ld_d=16), dict(kind=7), dict(logits=0), dict(ids=0), dict(counts=0), dict(out=0),
                                 dict(ld=7), dict(ld_d=7), dict(ld_d=1 << 24), dict(T=-1), dict(out=2 * P + 2), dict(dg=P + 1), dict(dl=P + 2),
                                 dict(out=P, ld=9)])
def test_route_backward_refuses(bad):
    assert back(**bad) == EINVAL


def test_route_backward_of_nothing():
    assert back(T=0, logits=0, ids=0, counts=0, out=0) == OK


def test_binding_refuses_what_the_library_cannot_see():
    """Host tensors, wrong types, inner strides, buffers that are too small: ValueError before the library is called."""
    x = torch.zeros((4, 64), dtype=torch.bfloat16)
    b = torch.zeros(4096, dtype=torch.uint8)
    with pytest.raises(ValueError):
        sm.mx_quantize(x, b, b, 0)                                # not on the GPU
    with pytest.raises(ValueError):
        sm.mx_gemm(x.float(), None, b, b, None, x, 0)
    with pytest.raises(ValueError):
        sm.route(x, torch.zeros((4, 1), dtype=torch.int32), b, b, b, b, 0)
    with pytest.raises(ValueError):
        sm.route_backward(x, torch.zeros((4, 1), dtype=torch.int32), b, x, 0)
