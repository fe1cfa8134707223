"""Products of few rows whose tiles of 32 x 32 are more than an XCD's runs of 64 hold (512): every tile has to be somebody's.  Values are small whole numbers, so that
products and sums are exact in fp32 and results equal to the bit; results hold another value first."""
import pytest
import torch

import paper_2310_18859_amd as sm
from paper_2310_18859_amd.moe_layer import MoELayer

pytestmark = pytest.mark.gpu
BF, F32 = torch.bfloat16, torch.float32

# groups' rows, columns of the result, length of the sum: what decoding and small batches have, and tiles around 512 and 1024
SIZES = [([1, 1, 1, 1, 1, 0, 0, 0], 4096, 4096), ([1, 0, 1, 1, 1, 1, 0, 1], 4096, 4096), ([1] * 6, 4096, 14336), ([0, 1, 0, 0, 0, 0, 1] * 4 + [1] + [0] * 35, 2048, 4096),
         ([1], 28672, 8192), ([1], 16640, 4096), ([1, 0, 1] * 12 + [0] * 28, 1024, 4096), ([40, 0, 33, 1], 4096, 4096), ([1, 1], 8192, 2080), ([1, 1, 1], 5464, 2064),
         ([1, 1], 8216, 2080), ([1], 32776, 8192), ([2, 3], 20480, 8192)]


def whole(shape, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randint(-3, 4, shape, generator=g, device="cuda", dtype=torch.int8).to(BF)


@pytest.mark.parametrize("counts,cols,length", SIZES)
@pytest.mark.parametrize("job", ["product", "input"])
def test_every_tile_is_written(counts, cols, length, job):
    at = [0]
    for n in counts:
        at.append(at[-1] + n)
    M, G = at[-1], len(counts)
    offsets = torch.tensor(at, dtype=torch.int32, device="cuda")
    rows = whole((M, length), cols + length)
    w = whole((G, cols, length) if job == "product" else (G, length, cols), cols)
    want = torch.zeros((M, cols), device="cuda", dtype=torch.float64)
    for g in range(G):
        if counts[g]:
            want[at[g]:at[g + 1]] = rows[at[g]:at[g + 1]].double() @ (w[g].double().t().contiguous() if job == "product" else w[g].double())
    for dtype in (F32, BF):
        out = torch.full((M, cols), 77.0, dtype=dtype, device="cuda")
        if job == "product":
            bias, pre = torch.arange(G * cols, device="cuda", dtype=F32).view(G, cols) % 5, torch.full((M, cols), 77.0, dtype=BF, device="cuda")
            sm.expert_gemm(rows, w, offsets, out, torch.cuda.current_stream(), bias=bias, activation=sm.ACT_RELU, pre=pre)
            v = want + bias[torch.repeat_interleave(torch.arange(G, device="cuda"), torch.tensor(counts, device="cuda"))]
            assert torch.equal(pre, v.to(BF))
            assert torch.equal(out, v.clamp_min(0).to(dtype))
        else:
            sm.expert_gemm_input(rows, w, offsets, out, torch.cuda.current_stream())
            assert torch.equal(out, want.to(dtype))


def test_decoding_batch_through_the_layer():
    """24 tokens over 64 experts: the second product and the rows' gradient of the first have 768 tiles.  Every value is read back through buffers of NaN; the sums
    are off by a step of bf16 of the largest value at most, as the hidden values, the experts' results and their gradients are rounded to it."""
    T, E, d, F = 24, 64, 1024, 4096
    g = torch.Generator(device="cuda").manual_seed(3)
    x, dy = (torch.randn((T, d), generator=g, device="cuda").to(BF) for _ in range(2))
    w_in, w_out = ((torch.randn(s, generator=g, device="cuda") * s[2] ** -0.5).to(BF) for s in ((E, F, d), (E, d, F)))
    to = torch.randperm(E, generator=g, device="cuda")[:T]
    logits = torch.full((T, E), -9.0, device="cuda")
    logits[torch.arange(T, device="cuda"), to] = 9.0
    layer = MoELayer(E, d, F, T, activation="none")
    for t in (layer.x_rows, layer.y_rows, layer.pre, layer.h):
        t.fill_(float("nan"))
    y, _ = layer.forward(x, logits, w_in, w_out)
    dx = layer.backward(dy, logits, w_in, w_out)["dx"]
    gate = layer.gates.double()
    for t in range(T):
        a, b = w_in[to[t]].double(), w_out[to[t]].double()
        h = (a @ x[t].double()).to(BF).double()
        want = (b @ h).to(BF).double() * gate[t]
        back = (dy[t].double() * gate[t]).to(BF).double()
        want_dx = ((back @ b).to(BF).double() @ a).to(BF).double()
        for got, of in ((y[t], want), (dx[t], want_dx)):
            assert (got.double() - of).abs().max() <= 2.0 ** -7 * of.abs().max()
