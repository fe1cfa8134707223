"""Tokens that take no part in a routed layer: their rows of y are 0 whatever they hold, and nobody else sees them."""
import numpy as np
import pytest
import torch

import paper_2310_18859_amd as sm
from paper_2310_18859_amd.mx_layer import MxMoELayer

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
E, D, F = 8, 256, 384


def made(T, k, x4, seed=1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    normal = lambda *s: torch.randn(s, generator=g, device=DEV)  # noqa: E731
    layer = MxMoELayer(E, D, F, T, top_k=k, normalize=True, tokens_in_4_bits=x4)
    layer.load_experts(normal(E, F, D).mul_(0.08).bfloat16(), normal(E, D, F).mul_(0.08).bfloat16())
    return layer, normal(T, D).bfloat16(), normal(T, E) * 2, normal(T, D).bfloat16()


@pytest.mark.parametrize("x4", [False, True])
@pytest.mark.parametrize("T,k", [(5, 1), (150, 1), (150, 3), (300, 2)])
def test_what_is_no_number_in_masked_rows(T, k, x4):
    """Infinities, NaN and values whose products overflow in masked rows, and in rows whose logits are all -infinity.  The others' results
    are bit for bit those of a batch whose masked rows hold ordinary values."""
    layer, x, logits, dy = made(T, k, x4)
    mask = torch.arange(T, device=DEV) % 3 != 1
    logits[torch.arange(T, device=DEV) % 6 == 3] = float("-inf")
    part = mask & (torch.arange(T, device=DEV) % 6 != 3)
    one = torch.ones(1, device=DEV)
    want, want_loss = (t.clone() for t in layer.forward(x, logits, mask))
    want_grad = layer.router_gradient(logits, dy, one, mask)
    assert (want[~part] == 0).all() and (want[part] != 0).any(1).all() and (want_grad[~part] == 0).all()
    out = torch.nonzero(~part)[:, 0]
    for value in (float("nan"), float("inf"), float("-inf"), 3e38):
        bad, bad_logits, bad_dy = x.clone(), logits.clone(), dy.clone()
        bad[out], bad_dy[out] = value, value
        bad[out[::2], 7:] = 1.0                                        # one value is enough
        bad_logits[torch.nonzero(~mask)[:, 0]] = value
        y, loss = layer.forward(bad, bad_logits, mask)
        assert torch.equal(y, want) and torch.equal(loss, want_loss)
        assert torch.equal(layer.router_gradient(bad_logits, bad_dy, one, mask), want_grad)
    layer.close()


@pytest.mark.parametrize("T,d,k", [(1, 128, 1), (77, 128, 1), (50, 768, 3), (33, 256, 8)])
def test_combine_routed(T, d, k):
    """Rows with a gate that is not 0, a NaN one among them, are those of the plain combine; rows without are 0 and are not read."""
    g = torch.Generator(device=DEV).manual_seed(T)
    pairs = T * k
    ctx = sm.Context(1, E, d, 128, 1, 1, pairs)
    ctx.set_top_k(k)
    ws = torch.zeros(ctx.workspace_bytes(pairs), dtype=torch.uint8, device=DEV)
    lay = ctx.workspace_layout(pairs)
    rows = ws[lay.y_perm:lay.y_perm + pairs * d * 2].view(torch.bfloat16).view(pairs, d)
    inv = ws[lay.inv:lay.inv + pairs * 4].view(torch.int32)
    rows.copy_(torch.randn((pairs, d), generator=g, device=DEV))
    inv.copy_(torch.randperm(pairs, generator=g, device=DEV))
    gates = torch.rand((T, k), generator=g, device=DEV) + 0.1
    gates[torch.rand((T, k), generator=g, device=DEV) < 0.3] = 0
    gates[1::7] = 0
    gates[2::7] = -0.0
    gates[3::7, k - 1] = float("nan")
    gates[4::7] = 0
    gates[4::7, k - 1] = 1e-40                                         # small, but a part
    none = (gates == 0).all(1)
    rows[inv.view(T, k)[none].long().flatten()] = float("nan")
    plain, routed = (torch.full((T + 1, d), 77.0, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    ctx.combine(gates, pairs, plain, ws, torch.cuda.current_stream())
    ctx.combine_routed(gates, pairs, routed, ws, torch.cuda.current_stream())
    bits = lambda t: t.view(torch.int16).cpu().numpy()  # noqa: E731
    assert np.array_equal(bits(plain[:T][~none]), bits(routed[:T][~none]))
    assert (bits(routed[:T][none]) == 0).all() and torch.isnan(plain[:T][none]).all()
    assert (routed[T] == 77).all()
    ctx.close()


def test_combine_routed_refuses():
    ctx = sm.Context(1, E, 128, 128, 1, 1, 16)
    ctx.set_top_k(2)
    ws = torch.zeros(ctx.workspace_bytes(16), dtype=torch.uint8, device=DEV)
    gates, y = torch.zeros(16, device=DEV), torch.zeros((8, 128), dtype=torch.bfloat16, device=DEV)
    for g, T, out, w in ((None, 16, y, ws), (gates, 16, None, ws), (gates, 15, y, ws), (gates, 18, y, ws), (gates, -2, y, ws), (gates, 16, y, ws[256:])):
        with pytest.raises(sm.SidaError):
            ctx.combine_routed(g, T, out, w, torch.cuda.current_stream())
    ctx.combine_routed(None, 0, None, ws, torch.cuda.current_stream())
    ctx.close()
