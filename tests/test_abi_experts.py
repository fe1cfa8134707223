"""What the operators of plain bf16 experts refuse, before anything is enqueued: no GPU is needed."""
import ctypes as C

import pytest
import torch

import paper_2310_18859_amd as sm

OK, EINVAL, ENOSPC = 0, -1, -2
P = 1 << 20                                                       # an aligned address that is never followed


def sort(E=8, k=2, ids=P, gates=0, T=5, offsets=P, places=P, ws=P, n=1 << 20):
    return sm.lib().sida_expert_sort(E, k, ids, gates, T, offsets, places, ws, n, 0)


@pytest.mark.parametrize("bad", [dict(E=0), dict(E=257), dict(k=0), dict(k=9), dict(T=-1), dict(T=1 << 25), dict(ids=0), dict(offsets=0), dict(places=0), dict(ws=0),
                                 dict(ids=P + 2), dict(gates=P + 1), dict(offsets=P + 2), dict(places=P + 1), dict(ws=P + 2)])
def test_sort_refuses(bad):
    assert sort(**bad) == EINVAL


def test_sort_workspace():
    for T, chunks in ((0, 1), (1, 1), (2048, 1), (2049, 3), (1 << 18, 256), ((1 << 25) - 1, 256)):
        n = sm.expert_sort_workspace_bytes(64, 2, T)
        assert n == chunks * 256
        assert sort(E=64, T=T, n=n - 1) == ENOSPC
    for bad in ((0, 1, 5), (257, 1, 5), (8, 9, 5), (8, 1, -1), (8, 2, 1 << 25), (8, 1, 1 << 40), (1 << 33, 1, 5)):
        assert sm.expert_sort_workspace_bytes(*bad) == 0


def cfg_rows(T=5, k=2, M=10, d=64, kind=sm.BF16, cfg=True):
    return C.byref(sm.SidaExpertRowsConfig(T, k, M, d, kind)) if cfg else None


def rows(x=P, ld_x=64, places=P, rows=P, ld_rows=64, **c):
    return sm.lib().sida_expert_rows(cfg_rows(**c), x, ld_x, places, rows, ld_rows, 0)


def total(rows=P, ld_rows=64, places=P, gates=0, res=0, ld_res=64, y=P, ld_y=64, **c):
    return sm.lib().sida_expert_sum(cfg_rows(**c), rows, ld_rows, places, gates, res, ld_res, y, ld_y, 0)


def back(dy=P, ld_dy=64, rows=P, ld_rows=64, places=P, gates=0, d_rows=P, ld_d=64, dg=P, **c):
    return sm.lib().sida_expert_sum_backward(cfg_rows(**c), dy, ld_dy, rows, ld_rows, places, gates, d_rows, ld_d, dg, 0)


CFG = [dict(cfg=False), dict(T=-1), dict(k=0), dict(k=9), dict(T=1 << 25), dict(M=-1), dict(d=0), dict(d=65537), dict(kind=sm.MXFP4), dict(kind=-1), dict(places=0),
       dict(places=P + 2)]


@pytest.mark.parametrize("bad", CFG + [dict(x=0), dict(x=P + 1), dict(x=P + 2, kind=sm.FP32), dict(ld_x=63), dict(ld_x=1 << 24), dict(rows=0), dict(rows=P + 1),
                                       dict(ld_rows=63), dict(ld_rows=1 << 24)])
def test_rows_refuse(bad):
    assert rows(**bad) == EINVAL


@pytest.mark.parametrize("bad", CFG + [dict(rows=0), dict(rows=P + 1), dict(ld_rows=63), dict(y=0), dict(y=P + 1), dict(ld_y=63), dict(ld_y=1 << 24), dict(gates=P + 2),
                                       dict(res=P + 1), dict(res=2 * P, ld_res=63), dict(res=P, ld_res=72)])
def test_sum_refuses(bad):
    assert total(**bad) == EINVAL


@pytest.mark.parametrize("bad", CFG + [dict(dy=0), dict(dy=P + 1), dict(ld_dy=63), dict(rows=0), dict(rows=P + 1), dict(ld_rows=63), dict(d_rows=0), dict(d_rows=P + 1),
                                       dict(ld_d=63), dict(ld_d=1 << 24), dict(dg=P + 2), dict(gates=P + 2), dict(ld_d=72)])
def test_sum_backward_refuses(bad):
    assert back(**bad) == EINVAL


def test_rows_of_nothing():
    assert rows(T=0, x=0, places=0, rows=0) == OK and rows(M=0, x=0, places=0, rows=0) == OK
    assert total(T=0, rows=0, places=0, y=0) == OK and back(T=0, dy=0, rows=0, places=0, d_rows=0, dg=0) == OK


def cfg_gemm(groups=2, N=64, K=72, out=sm.BF16, act=0, cfg=True):
    return C.byref(sm.SidaExpertGemmConfig(groups, N, K, out, act)) if cfg else None


def gemm(x=P, ldx=72, M=5, w=P, offsets=P, bias=0, pre=0, ld_pre=64, res=0, ld_res=64, y=P, ldy=64, **c):
    return sm.lib().sida_expert_gemm(cfg_gemm(**c), x, ldx, M, w, offsets, bias, pre, ld_pre, res, ld_res, y, ldy, 0)


def gemm_input(dy=P, ld_dy=64, M=5, w=P, offsets=P, pre=2 * P, ld_pre=72, dx=P, ld_dx=72, **c):
    return sm.lib().sida_expert_gemm_input(cfg_gemm(**c), dy, ld_dy, M, w, offsets, pre, ld_pre, dx, ld_dx, 0)


def gemm_weights(dy=P, ld_dy=64, x=P, ldx=72, M=5, offsets=P, dw=P, db=0, ws=P, n=1 << 28, **c):
    return sm.lib().sida_expert_gemm_weights(cfg_gemm(**c), dy, ld_dy, x, ldx, M, offsets, dw, db, ws, n, 0)


GEMM = [dict(cfg=False), dict(groups=0), dict(groups=257), dict(N=0), dict(N=60), dict(N=65544), dict(K=0), dict(K=12), dict(K=65544), dict(N=65536, K=65536),
        dict(groups=256, N=32768, K=32768), dict(out=sm.MXFP4), dict(act=-1), dict(act=4), dict(M=-1), dict(M=(1 << 24) + 1), dict(offsets=0), dict(offsets=P + 2)]


@pytest.mark.parametrize("bad", GEMM + [dict(M=1 << 24, N=4096, ldy=4096), dict(x=0), dict(x=P + 8), dict(ldx=64), dict(ldx=76), dict(ldx=(1 << 22) + 8), dict(w=0), dict(w=P + 8),
                                        dict(y=0), dict(y=P + 8), dict(ldy=56), dict(ldy=68), dict(ldy=66, out=sm.FP32), dict(ldy=(1 << 21) + 4, out=sm.FP32), dict(ldy=1 << 62), dict(ldy=(1 << 22) + 8), dict(bias=P + 4),
                                        dict(pre=P + 8), dict(pre=2 * P, ld_pre=56), dict(res=P + 8), dict(res=2 * P, ld_res=56), dict(res=P, ld_res=72)])
def test_gemm_refuses(bad):
    assert gemm(**bad) == EINVAL


@pytest.mark.parametrize("bad", GEMM + [dict(dy=0), dict(dy=P + 8), dict(ld_dy=56), dict(ld_dy=68), dict(w=0), dict(w=P + 8), dict(dx=0), dict(dx=P + 8), dict(ld_dx=64), dict(ld_dx=76),
                                        dict(pre=0, act=sm.ACT_GELU), dict(pre=P + 8), dict(ld_pre=64), dict(ld_pre=76), dict(pre=P, ld_dx=80), dict(pre=P, out=sm.FP32)])
def test_gemm_input_refuses(bad):
    assert gemm_input(**bad) == EINVAL


@pytest.mark.parametrize("bad", GEMM[:-3] + [dict(act=sm.ACT_RELU), dict(M=-1), dict(offsets=0), dict(offsets=P + 2), dict(dy=0), dict(dy=P + 8), dict(ld_dy=56), dict(x=0),
                                             dict(x=P + 8), dict(ldx=64), dict(dw=0), dict(dw=P + 8), dict(db=P + 2), dict(ws=P + 8)])
def test_gemm_weights_refuses(bad):
    assert gemm_weights(**bad) == EINVAL


def test_gemm_weights_workspace():
    """Many rows into small matrices are summed in parts; what is enough for them is enough for fewer."""
    for groups, N, K in ((4, 520, 264), (1, 1024, 1024), (1, 8, 8), (3, 128, 512)):
        cfg, before = sm.SidaExpertGemmConfig(groups, N, K, sm.FP32, 0), 0
        for M in (0, 1, 100, 512, 1000, 4097, 16385, 70000, 1 << 20):
            n = sm.expert_gemm_weights_workspace_bytes(cfg, M)
            assert n >= before
            before = n
            if n:
                call = dict(groups=groups, N=N, K=K, M=M, ld_dy=N, ldx=K, out=sm.FP32)
                assert gemm_weights(**call, n=n - 1) == ENOSPC and gemm_weights(**call, ws=0) == EINVAL
        assert before
    assert sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(64, 4096, 1024, sm.BF16, 0), 1 << 20) == 0
    assert sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(4, 521, 264, sm.BF16, 0), 5) == 0
    assert sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(4, 520, 264, sm.BF16, 0), -1) == 0


def test_gemm_of_nothing():
    assert gemm(M=0, x=0, y=0, w=0, offsets=0) == OK and gemm_input(M=0, dy=0, dx=0, w=0, offsets=0) == OK


def test_binding_refuses_what_the_library_cannot_see():
    """Host tensors, wrong types and shapes: ValueError before the library is called."""
    x, b, p = torch.zeros((4, 64), dtype=torch.bfloat16), torch.zeros(4096, dtype=torch.uint8), torch.zeros((4, 1), dtype=torch.int32)
    o = torch.zeros(9, dtype=torch.int32)
    for call in (lambda: sm.expert_sort(p, o, p, b, 0), lambda: sm.expert_rows(x, p, x, 0), lambda: sm.expert_sum(x, p, x, 0),
                 lambda: sm.expert_sum_backward(x, x, p, x, 0), lambda: sm.expert_gemm(x, x, None, x, 0), lambda: sm.expert_gemm_input(x, x, None, x, 0),
                 lambda: sm.expert_gemm_weights(x, x, None, x, b, 0)):
        with pytest.raises(ValueError):
            call()
