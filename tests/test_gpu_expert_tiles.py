"""The experts' products at sizes that reach each of their kernels (which one a size reaches is checked on the host, tests/test_expert_rule_host.py), with groups
whose last tiles have every number of 32-row blocks.  Values are small whole numbers: products and sums are exact in fp32, and results the oracle's, to the bit."""
import pytest
import torch

import paper_2310_18859_amd as sm

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# kernel, groups' rows, columns of the result, length of the sum.  The sums: whole stages of 64, a part of the last one, fewer than a ring's stages, one only.
RAGGED = [300, 1, 0, 131, 64, 33, 97, 15]
SIZES = (
    [("few", [1], n, c) for n, c in ((8, 8), (40, 64), (136, 1000), (1024, 4096))] + [("few", [3, 0, 1, 33, 64], n, c) for n, c in ((72, 520), (104, 2056))]
    + [("rows32", [9, 1, 0, 33, 64, 70, 5, 2] * 2, n, c) for n, c in ((520, 64), (1032, 8), (648, 200), (904, 712))] + [("rows32", [500], 1024, 328)]
    + [("rows64", [41, 1, 0, 64, 65, 33, 96, 128] * 6, n, c) for n, c in ((520, 64), (648, 136), (1288, 8), (520, 776))]
    + [("square128", RAGGED + [128, 90, 129, 255, 256] * 3, n, c) for n, c in ((1032, 64), (1160, 200), (904, 520), (1288, 8), (2056, 328))]
    + [("rows256", [480 + 32 * i + (i * 7) % 32 for i in range(9)] * 3, n, c) for n, c in ((1800, 64), (2056, 200), (1544, 328), (1800, 136), (1544, 16))]
    # one group, whose rows of tiles are walked four at a time, with one to three left over
    + [("rows32", [300], 1600, 72), ("square128", [700], 4360, 136), ("square128", [590], 5640, 64), ("rows256", [4648], 3848, 72), ("rows256", [4200], 4104, 200)]
)


def whole(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda").to(BF)


def groups_of(counts):
    bounds = [0]
    for n in counts:
        bounds.append(bounds[-1] + n)
    return bounds, torch.tensor(bounds, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("kernel,counts,cols,length", SIZES)
@pytest.mark.parametrize("job", ["product", "input"])
def test_rows(kernel, counts, cols, length, job):
    at, offsets = groups_of(counts)
    M, G = at[-1], len(counts)
    rows = whole((M, length), cols + length)
    w = whole((G, cols, length) if job == "product" else (G, length, cols), cols)
    want = torch.zeros((M, cols), device="cuda")
    for g in range(G):
        if counts[g]:
            want[at[g]:at[g + 1]] = rows[at[g]:at[g + 1]].float() @ (w[g].float().t().contiguous() if job == "product" else w[g].float())
    for dtype in (F32, BF):
        out = torch.full((M, cols + 8), 77.0, dtype=dtype, device="cuda")
        if job == "product":
            bias, pre = torch.arange(G * cols, device="cuda", dtype=F32).view(G, cols) % 5, torch.full((M, cols), 77.0, dtype=BF, device="cuda")
            sm.expert_gemm(rows, w, offsets, out[:, :cols], torch.cuda.current_stream(), bias=bias, activation=sm.ACT_RELU, pre=pre, residual=None)
            group = torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(counts, device="cuda"))
            v = want + bias[group]
            assert torch.equal(pre, v.to(BF))
            assert torch.equal(out[:, :cols], v.clamp_min(0).to(dtype))
        else:
            sm.expert_gemm_input(rows, w, offsets, out[:, :cols], torch.cuda.current_stream())
            assert torch.equal(out[:, :cols], want.to(dtype))
        assert out[:, cols:].eq(77).all()


# kernel, groups' rows, N, K
WEIGHTS = (
    [("rows256", RAGGED, N, K) for N, K in ((2056, 1032), (1800, 1800))] + [("rows256", [0, 5, 64, 65, 200, 129, 1, 700], 2048, 1024)]
    + [("square128", RAGGED, N, K) for N, K in ((136, 264), (520, 72), (648, 648))] + [("square128", [70, 0, 3], 8, 8)]
    + [("parts", [2500, 0, 3, 700], N, K) for N, K in ((136, 264), (520, 72), (8, 8), (264, 392))] + [("parts", [9000], 1032, 520)]
)


@pytest.mark.parametrize("kernel,counts,N,K", WEIGHTS)
@pytest.mark.parametrize("bias", [False, True])
def test_weights(kernel, counts, N, K, bias):
    at, offsets = groups_of(counts)
    M, G = at[-1], len(counts)
    dy, x = whole((M, N), N), whole((M, K), K + 1)
    want = torch.stack([dy[a:b].float().t().contiguous() @ x[a:b].float() for a, b in zip(at[:-1], at[1:])])
    for dtype, kind in ((F32, sm.FP32), (BF, sm.BF16)):
        ws = torch.full((max(16, sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(G, N, K, kind, 0), M)),), 255, dtype=torch.uint8, device="cuda")
        dw, db = torch.full((G, N, K), 77.0, dtype=dtype, device="cuda"), torch.full((G, N), 77.0, device="cuda")
        sm.expert_gemm_weights(dy, x, offsets, dw, ws, torch.cuda.current_stream(), d_bias=db if bias else None)
        assert torch.equal(dw, want.to(dtype))
        if bias:
            assert torch.equal(db, torch.stack([dy[a:b].float().sum(0) for a, b in zip(at[:-1], at[1:])]))
        else:
            assert db.eq(77).all()


def test_calls_at_once():
    """Two streams, each with a workspace of its own."""
    at, offsets = groups_of([3000, 1000])
    dy, x, w = whole((4000, 264), 1), whole((4000, 136), 2), whole((2, 264, 136), 3)
    need = sm.expert_gemm_weights_workspace_bytes(sm.SidaExpertGemmConfig(2, 264, 136, sm.FP32, 0), 4000)
    assert need > 0
    want = torch.stack([dy[a:b].float().t().contiguous() @ x[a:b].float() for a, b in zip(at[:-1], at[1:])])
    want_y = torch.cat([x[a:b].float() @ w[g].float().t().contiguous() for g, (a, b) in enumerate(zip(at[:-1], at[1:]))])
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    out = []
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            ws, dw, y = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.empty((2, 264, 136), device="cuda"), torch.empty((4000, 264), device="cuda")
            sm.expert_gemm_weights(dy, x, offsets, dw, ws, streams[i % 2])
            sm.expert_gemm(x, w, offsets, y, streams[i % 2])
            out.append((ws, dw, y))
    torch.cuda.synchronize()
    assert all(torch.equal(dw, want) and torch.equal(y, want_y) for _, dw, y in out)
