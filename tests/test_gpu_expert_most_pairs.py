"""The gradient of the weighted sum with the most pairs that a call takes, 2^26 - 1 of them, nearly all without a part: a launch of as many lanes as fit."""
import pytest
import torch

import paper_2310_18859_amd as sm

pytestmark = pytest.mark.gpu


def test_gradient_of_the_sum():
    T, k, d, M = ((1 << 26) - 1) // 3, 3, 512, 8
    assert T * k == (1 << 26) - 1
    pairs = torch.tensor([0, 1, 2, 12345, T * k // 2, T * k - 3, T * k - 2, T * k - 1], device="cuda")
    places = torch.full((T, k), -1, dtype=torch.int32, device="cuda")
    places.view(-1)[pairs] = torch.arange(M, dtype=torch.int32, device="cuda")
    dy = torch.empty((T, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(1)
    dy[pairs // k] = torch.randint(-3, 4, (M, d), generator=g, device="cuda").to(torch.bfloat16)
    rows = torch.randint(-3, 4, (M, d), generator=g, device="cuda").to(torch.bfloat16)
    d_rows, d_gates = torch.full((M, d), 77.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, k), 77.0, device="cuda")
    sm.expert_sum_backward(dy, rows, places, d_rows, torch.cuda.current_stream(), d_gates=d_gates)
    assert torch.equal(d_rows, dy[pairs // k])
    assert torch.equal(d_gates.view(-1)[pairs], (dy[pairs // k].float() * rows.float()).sum(1))   # whole numbers: exact
    d_gates.view(-1)[pairs] = 0
    assert not d_gates.any()
