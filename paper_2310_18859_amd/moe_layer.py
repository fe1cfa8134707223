"""A routed MoE layer around plain bf16 experts that can be trained: the router's choice, tokens to their experts, the experts' two
products, the weighted sum, and the way back through all of them.  Buffers and streams only; the arithmetic is the library's."""
from __future__ import annotations

import torch

from .binding import (ACT_GELU, ACT_NONE, ACT_RELU, ACT_SILU, BF16, FP32, SidaExpertGemmConfig, SidaRouteConfig, expert_gemm, expert_gemm_input,
                      expert_gemm_weights, expert_gemm_weights_workspace_bytes, expert_rows, expert_sort, expert_sort_workspace_bytes, expert_sum,
                      expert_sum_backward, route, route_backward, route_workspace_bytes)
from .mx_layer import MxMoELayer

ACTIVATIONS = {"none": ACT_NONE, "relu": ACT_RELU, "gelu": ACT_GELU, "silu": ACT_SILU}
MOST_EXPERTS, MOST_TOP_K, MOST_WIDTH = 256, 8, 65536                       # of the library's calls, as are the limits of pairs in `forward`


class MoELayer:
    """y[t,:] = residual[t,:] + sum_j gates[t,j] * (W_out[e] act(W_in[e] x[t,:] + b_in[e]) + b_out[e]), e = ids[t,j] the top_k experts of logits[t,:].

    The parameters are the caller's: w_in bf16 [E, d_ff, d_model], w_out bf16 [E, d_model, d_ff], and b_in fp32 [E, d_ff], b_out fp32 [E, d_model] or None;
    d_model and d_ff are multiples of 8.  A token that is masked, or whose logits are all -infinity, goes to no expert and costs nothing.
    Streams and devices are as those of MxMoELayer: everything is enqueued on `stream`, behind what torch's current stream has been given when a call is
    made, and the current stream goes on behind the call.  y and the gradients that `backward` returns are new tensors; the loss, ids, gates and counts are
    views of the layer's buffers and hold until its next forward call, as does what `backward` needs of the forward call."""

    def __init__(self, E, d_model, d_ff, max_tokens, top_k=1, normalize=False, activation="gelu", device="cuda:0", stream=None):
        if activation not in ACTIVATIONS:
            raise ValueError(f"activation: one of {sorted(ACTIVATIONS)} is needed, not {activation!r}")
        if d_model % 8 or d_ff % 8:
            raise ValueError(f"d_model and d_ff: multiples of 8 are needed, not {d_model} and {d_ff}")
        if not (1 <= E <= MOST_EXPERTS and 1 <= top_k <= min(E, MOST_TOP_K) and 8 <= d_model <= MOST_WIDTH and 8 <= d_ff <= MOST_WIDTH and
                d_model * d_ff <= 1 << 30 and E * d_model * d_ff <= 1 << 36 and 0 <= max_tokens * top_k < 1 << 26):
            raise ValueError(f"sizes that the experts' products take are needed, not {E} experts of {d_model} x {d_ff}, {top_k} to a token, {max_tokens} tokens")
        self.dev = torch.device(device)
        if self.dev.type == "cuda" and self.dev.index is None:
            self.dev = torch.device("cuda", torch.cuda.current_device())
        self.E, self.d, self.F, self.k, self.normalize, self.act = E, d_model, d_ff, top_k, normalize, ACTIVATIONS[activation]
        self.max_tokens, self.tokens = max_tokens, None                    # tokens of the last forward call
        if stream is None:
            stream = torch.cuda.current_stream(self.dev)
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=self.dev) if stream else torch.cuda.default_stream(self.dev)
        self.stream = stream
        with self._on_stream():                                            # the buffers' memory is that stream's
            self._make_buffers()

    _on_stream, _need = MxMoELayer._on_stream, MxMoELayer._need

    def _new(self, *shape, dtype=torch.bfloat16):
        return torch.empty(shape, dtype=dtype, device=self.dev)

    def _make_buffers(self):
        T, pairs = self.max_tokens, self.max_tokens * self.k
        self.route_ws = self._new(max(route_workspace_bytes(SidaRouteConfig(self.E, self.k, t, 0), T) for t in (BF16, FP32)), dtype=torch.uint8)
        self.sort_ws = self._new(expert_sort_workspace_bytes(self.E, self.k, T), dtype=torch.uint8)
        self.ids, self.gates = self._new(T, self.k, dtype=torch.int32), self._new(T, self.k, dtype=torch.float32)
        self.counts, self.loss = self._new(self.E, dtype=torch.int32), self._new(1, dtype=torch.float32)
        self.offsets, self.places = self._new(self.E + 1, dtype=torch.int32), self._new(T, self.k, dtype=torch.int32)
        self.x_rows, self.y_rows = self._new(pairs, self.d), self._new(pairs, self.d)
        self.pre, self.h = self._new(pairs, self.F), self._new(pairs, self.F)

    # What the library's calls refuse is refused here, before the first of them: the later ones would leave the buffers half overwritten.
    def _matrix(self, t, what, shape, dtypes=(torch.bfloat16,)):
        self._need(t, what, shape, dtypes)
        rows, cols = shape
        if t.numel() and ((cols > 1 and t.stride(1) != 1) or (rows > 1 and not cols <= t.stride(0) < 1 << 24)):
            raise ValueError(f"{what}: contiguous rows, one behind the other and less than 2^24 values apart, are needed, not strides {t.stride()}")

    def _values(self, t, what, n, dtypes):
        """At least n values one after the other, or None."""
        if t is not None and (t.dtype not in dtypes or t.numel() < n or not t.is_contiguous() or t.device != self.dev):
            raise ValueError(f"{what}: a contiguous tensor of at least {n} values of {' or '.join(str(d) for d in dtypes)} on {self.dev} is needed")

    def _parameters(self, w_in, w_out, b_in, b_out):
        for t, what, shape, dtype in ((w_in, "w_in", (self.E, self.F, self.d), torch.bfloat16), (w_out, "w_out", (self.E, self.d, self.F), torch.bfloat16),
                                      (b_in, "b_in", (self.E, self.F), torch.float32), (b_out, "b_out", (self.E, self.d), torch.float32)):
            if t is not None or what[0] == "w":
                self._need(t, what, shape, (dtype,))
                if not t.is_contiguous() or t.data_ptr() % 16:
                    raise ValueError(f"{what}: a contiguous tensor from a 16-byte boundary on is needed")

    def forward(self, x, logits, w_in, w_out, b_in=None, b_out=None, mask=None, residual=None):
        """x: bf16 [T, d_model]; logits: bf16 or fp32 [T, E]; mask: bool [T] or None; residual: bf16 [T, d_model] or None.  Returns y bf16 [T, d_model] and the
        balance loss [1]."""
        T = x.shape[0] if x.dim() else 0
        self._matrix(x, "x", (T, self.d))
        if T > self.max_tokens:
            raise ValueError(f"x: at most {self.max_tokens} tokens, not {T}")
        if T * self.k > 1 << 24 or T * self.k * max(self.d, self.F) > 1 << 35:
            raise ValueError(f"x: 2^24 pairs of token and expert and 2^35 values of their rows at most, not {T} tokens of {self.k} experts each")
        self._matrix(logits, "logits", (T, self.E), (torch.bfloat16, torch.float32))
        self._values(mask, "mask", T, (torch.bool, torch.uint8))
        if residual is not None:
            self._matrix(residual, "residual", (T, self.d))
        self._parameters(w_in, w_out, b_in, b_out)
        y, s = self._new(T, self.d), self.stream                           # memory of the caller's stream
        pairs, self.tokens = T * self.k, None                              # a call that fails on its way leaves nothing to go back through
        with self._on_stream((self.ids, self.gates, self.counts, self.loss)):
            ids, gates, places = self.ids[:T], self.gates[:T], self.places[:T]
            route(logits, ids, gates, self.counts, self.loss, self.route_ws, s, mask=mask, normalize=self.normalize)
            expert_sort(ids, self.offsets, places, self.sort_ws, s, gates=gates)   # the router's gates are 0 where a token takes no part
            if T:
                x_rows, y_rows, pre, h = (t[:pairs] for t in (self.x_rows, self.y_rows, self.pre, self.h))
                expert_rows(x, places, x_rows, s)
                expert_gemm(x_rows, w_in, self.offsets, h, s, bias=b_in, activation=self.act, pre=pre)
                expert_gemm(h, w_out, self.offsets, y_rows, s, bias=b_out)
                expert_sum(y_rows, places, y, s, gates=gates, residual=residual)
        self.tokens = T
        return y, self.loss

    def backward(self, dy, logits, w_in, w_out, d_loss=None, mask=None, biases=True, weights_dtype=torch.float32):
        """Gradients of the last forward call, whose logits, mask and parameters are given again: dy bf16 [T, d_model], d_loss fp32 [1] or None.
        Returns a dict of dx bf16 [T, d_model] (through the experts; the residual's is dy), d_logits as the logits, d_w_in and d_w_out of weights_dtype, and
        with `biases` d_b_in and d_b_out fp32."""
        T = self.tokens
        if T is None:
            raise RuntimeError("backward: there has been no forward call")
        self._matrix(dy, "dy", (T, self.d))
        self._matrix(logits, "logits", (T, self.E), (torch.bfloat16, torch.float32))
        self._values(mask, "mask", T, (torch.bool, torch.uint8))
        self._values(d_loss, "d_loss", 1, (torch.float32,))
        self._parameters(w_in, w_out, None, None)
        if weights_dtype not in (torch.float32, torch.bfloat16):
            raise ValueError(f"weights_dtype: {torch.float32} or {torch.bfloat16} is needed, not {weights_dtype}")
        out = {"dx": self._new(T, self.d), "d_logits": torch.empty_like(logits), "d_w_in": self._new(self.E, self.F, self.d, dtype=weights_dtype),
               "d_w_out": self._new(self.E, self.d, self.F, dtype=weights_dtype)}
        if biases:
            out["d_b_in"], out["d_b_out"] = self._new(self.E, self.F, dtype=torch.float32), self._new(self.E, self.d, dtype=torch.float32)
        pairs, s, kind = T * self.k, self.stream, FP32 if weights_dtype == torch.float32 else BF16
        with self._on_stream():
            places, gates = self.places[:T], self.gates[:T]
            x_rows, y_rows, pre, h = (t[:pairs] for t in (self.x_rows, self.y_rows, self.pre, self.h))
            d_rows, d_pre, d_gates = self._new(pairs, self.d), self._new(pairs, self.F), self._new(T, self.k, dtype=torch.float32)
            ws = self._new(max(expert_gemm_weights_workspace_bytes(SidaExpertGemmConfig(self.E, n, k, kind, ACT_NONE), pairs)
                               for n, k in ((self.F, self.d), (self.d, self.F))), dtype=torch.uint8)
            if T:
                expert_sum_backward(dy, y_rows, places, d_rows, s, gates=gates, d_gates=d_gates)
            expert_gemm_weights(d_rows, h, self.offsets, out["d_w_out"], ws, s, d_bias=out.get("d_b_out"))
            expert_gemm_input(d_rows, w_out, self.offsets, d_pre, s, pre=pre, activation=self.act)
            expert_gemm_weights(d_pre, x_rows, self.offsets, out["d_w_in"], ws, s, d_bias=out.get("d_b_in"))
            expert_gemm_input(d_pre, w_in, self.offsets, d_rows, s)        # of x's rows, in the place of those of y's
            if T:
                expert_sum(d_rows, places, out["dx"], s)
                route_backward(logits, self.ids[:T], self.counts, out["d_logits"], s, d_gates=d_gates, d_loss=d_loss, mask=mask, normalize=self.normalize)
        return out
