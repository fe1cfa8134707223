"""A routed MoE layer with experts in 4 bits: serve a batch, look at what rounding the weights costs, and train the router for balance.

    python examples/routed_layer_in_4_bits.py            (needs an MI355X and the built library)
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2310_18859_amd.mx_layer import MxMoELayer  # noqa: E402


def main(E=32, d=768, F=3072, T=2048, k=2, steps=40, lr=0.02):
    g = torch.Generator(device="cuda").manual_seed(0)
    normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
    w_in, w_out = (normal(E, F, d) * 0.02).bfloat16(), (normal(E, d, F) * 0.02).bfloat16()
    router = normal(E, d) * 0.02 + torch.linspace(1, -1, E, device="cuda")[:, None] * 0.01
    x = (normal(T, d) + 0.1).bfloat16()
    mask = torch.arange(T, device="cuda") % 128 < 120                  # sequences of 128 with 8 padded tokens

    layer = MxMoELayer(E, d, F, T, top_k=k, normalize=True)
    layer.load_experts(w_in, w_out)
    y, loss = layer.forward(x, x.float() @ router.t(), mask)
    plain = torch.zeros((T, d), device="cuda")                         # the same tokens through the bf16 weights
    for e in range(E):
        t, j = (layer.ids[:T] == e).nonzero(as_tuple=True)
        out = torch.relu(x[t].float() @ w_in[e].float().t()) @ w_out[e].float().t()
        plain.index_add_(0, t, layer.gates[t, j][:, None] * out)
    off = float((y.float() - plain).norm() / plain.norm())
    print(f"served {T} tokens, {k} of {E} experts each; 4-bit weights change the outputs by {off:.3f} of their norm", flush=True)

    one = torch.ones(1, device="cuda")
    for step in range(steps):                                          # the balance loss alone trains the router here
        logits = x.float() @ router.t()
        _, loss = layer.forward(x, logits, mask)
        if step % 10 == 0 or step == steps - 1:
            c = layer.counts
            print(f"step {step}: balance loss {float(loss):.4f}, tokens per expert {int(c.min())} .. {int(c.max())}", flush=True)
        d_logits = layer.router_gradient(logits, torch.zeros_like(x), one, mask)
        router -= lr * (d_logits.t() @ x.float())
    layer.close()
    return off, float(loss)


if __name__ == "__main__":
    main()
