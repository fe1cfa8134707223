"""A routed MoE layer whose experts are held in 4 bits: the router's choice, the sort, the two grouped products and the
combine, and the gradient that trains the router.  Buffers and streams only; the arithmetic is the library's."""
from __future__ import annotations

import contextlib

import torch

from .binding import (BF16, FP32, MX_TILES, Context, SidaRouteConfig, mx_codes_bytes, mx_gemm, mx_quantize, mx_scales_bytes,
                      route, route_backward, route_workspace_bytes)


class MxMoELayer:
    """y[t,:] = sum_j gates[t,j] * W_out[e] relu(W_in[e] x[t,:]), e = ids[t,j] the top_k experts of logits[t,:].

    The weights take 17/64 of their bf16 bytes.  tokens_in_4_bits: x and the hidden values are rounded to MXFP4 too, and
    multiplied in 4 bits.  Everything is enqueued on `stream` (a torch stream or a raw one; default: torch's current one when the layer is
    made).  It goes on behind what torch's current stream has been given when a call is made, and the current stream goes on behind the call, so that
    inputs, results and the memory of both are used as on the current stream alone.  `device` need not be the current one.  y and the gradient are new tensors; the loss, ids, gates
    and counts are views of the layer's buffers and hold until its next forward call."""

    def __init__(self, E, d_model, d_ff, max_tokens, top_k=1, normalize=False, tokens_in_4_bits=False, device="cuda:0", stream=None):
        self.dev = torch.device(device)
        if self.dev.type == "cuda" and self.dev.index is None:
            self.dev = torch.device("cuda", torch.cuda.current_device())
        self.loaded, self.tokens = False, 0                                # experts are there; tokens of the last forward call
        self.E, self.d, self.F, self.k, self.normalize, self.x4 = E, d_model, d_ff, top_k, normalize, tokens_in_4_bits
        self.max_tokens, self.max_pairs = max_tokens, max_tokens * top_k
        if stream is None:
            stream = torch.cuda.current_stream(self.dev)
        elif isinstance(stream, int):
            stream = torch.cuda.ExternalStream(stream, device=self.dev) if stream else torch.cuda.default_stream(self.dev)
        self.stream = stream
        with self._on_stream():                                            # the buffers' memory is that stream's
            self._make_buffers(E, d_model, d_ff, max_tokens, top_k)

    def _make_buffers(self, E, d_model, d_ff, max_tokens, top_k):
        self.ctx = Context(1, E, d_model, d_ff, 1, 1, self.max_pairs)      # sort and combine; its expert pool stays unbound
        self.ctx.set_top_k(top_k)
        self.workspace = self._buffer(max(256, self.ctx.workspace_bytes(self.max_pairs)))
        route_bytes = max(route_workspace_bytes(SidaRouteConfig(E, top_k, t, 0), max_tokens) for t in (BF16, FP32))
        self.route_ws = self._buffer(route_bytes)
        self.experts = [tuple(self._buffer(E * size(rows, cols, MX_TILES)) for size in (mx_codes_bytes, mx_scales_bytes))
                        for rows, cols in ((d_ff, d_model), (d_model, d_ff))]
        self.ids = torch.empty((max_tokens, top_k), dtype=torch.int32, device=self.dev)
        self.gates = torch.empty((max_tokens, top_k), device=self.dev)
        self.counts = torch.empty(E, dtype=torch.int32, device=self.dev)
        self.loss = torch.empty(1, device=self.dev)
        if self.x4:
            widest = max(d_model, d_ff)
            self.x_codes = self._buffer(self.max_pairs * widest // 2)
            self.x_scales = self._buffer(self.max_pairs * (-(-widest // 256) * 8))

    @contextlib.contextmanager
    def _on_stream(self, shown=()):
        """The layer's stream is torch's current one inside, and its device the current one: the library's calls go to that, and the default
        streams of all devices have the same raw value.  shown: tensors of the stream's memory that the caller goes on to use."""
        with torch.cuda.device(self.dev):
            caller = torch.cuda.current_stream(self.dev)
            if caller == self.stream:
                yield
                return
            self.stream.wait_stream(caller)
            try:
                with torch.cuda.stream(self.stream):
                    yield
            finally:
                caller.wait_stream(self.stream)
                for t in shown:
                    t.record_stream(caller)

    def _buffer(self, nbytes):
        return torch.empty(nbytes, dtype=torch.uint8, device=self.dev)

    # dispatch, combine and torch's operations take what they are given for the layer's own sizes: what a tensor has to be is checked here,
    # before anything is enqueued.  The rest is checked by the calls that take it.
    def _need(self, t, what, shape, dtypes=(torch.bfloat16, torch.float32)):
        if tuple(t.shape) != shape or t.dtype not in dtypes or t.device != self.dev:
            raise ValueError(f"{what}: {list(shape)} of {' or '.join(str(d) for d in dtypes)} on {self.dev} is needed, "
                             f"not {list(t.shape)} of {t.dtype} on {t.device}")

    def load_experts(self, w_in, w_out):
        """w_in: bf16 or fp32 [E, d_ff, d_model], w_out [E, d_model, d_ff], on the GPU: rounded to MXFP4 and laid out."""
        for w, what, shape in ((w_in, "w_in", (self.E, self.F, self.d)), (w_out, "w_out", (self.E, self.d, self.F))):
            self._need(w, what, shape)
        with self._on_stream():
            for w, (codes, scales) in zip((w_in, w_out), self.experts):
                mx_quantize(w.reshape(-1, w.shape[2]), codes, scales, self.stream, layout=MX_TILES)   # rows are multiples of 128
        self.loaded = True

    def _region(self, layout, name, dtype, shape):
        n = torch.empty((), dtype=dtype).element_size()
        for v in shape:
            n *= v
        at = getattr(layout, name)
        return self.workspace[at:at + n].view(dtype).view(shape)

    def _product(self, x, weights, offsets, y, relu):
        scales = None
        if self.x4:
            rows, cols = x.shape
            codes = self.x_codes[:rows * cols // 2].view(rows, cols // 2)
            scales = self.x_scales[:rows * (-(-cols // 256) * 8)]
            mx_quantize(x, codes, scales, self.stream)
            x = codes
        mx_gemm(x, scales, *weights, offsets, y, self.stream, relu=relu)

    def forward(self, x, logits, mask=None):
        """x: bf16 [T, d_model] (copied where it is not contiguous from a 16-byte boundary on); logits: bf16 or fp32 [T, E]; mask: bool [T] or
        None (y is 0 where a token is masked, or all its logits are -infinity, whatever its x holds).  Returns y [T, d_model] and the balance loss [1]; ids, gates and counts are the layer's."""
        T = x.shape[0] if x.dim() else 0
        self._need(x, "x", (T, self.d), (torch.bfloat16,))
        if T > self.max_tokens:
            raise ValueError(f"x: at most {self.max_tokens} tokens, not {T}")
        self._need(logits, "logits", (T, self.E))
        if T and not self.loaded:
            raise RuntimeError("load_experts has not been called")
        y = torch.empty((T, self.d), dtype=torch.bfloat16, device=self.dev)   # memory of the caller's stream
        with self._on_stream((self.ids, self.gates, self.counts, self.loss)):
            x = x.contiguous()
            self._forward(x.clone() if x.data_ptr() % 16 else x, logits, mask, y)
        self.tokens = T
        return y, self.loss

    def _forward(self, x, logits, mask, y):
        T, pairs = x.shape[0], x.shape[0] * self.k
        ids, gates = self.ids[:T], self.gates[:T]
        route(logits, ids, gates, self.counts, self.loss, self.route_ws, self.stream, mask=mask, normalize=self.normalize)
        if T == 0:
            return
        self.ctx.dispatch(x, ids, pairs, self.workspace, self.stream)
        lay = self.ctx.workspace_layout(pairs)
        offsets = self._region(lay, "offsets", torch.int32, (self.E + 1,))
        h = self._region(lay, "h", torch.bfloat16, (pairs, self.F))
        self.y_perm = self._region(lay, "y_perm", torch.bfloat16, (pairs, self.d))
        self.inv = self._region(lay, "inv", torch.int32, (pairs,))
        self._product(self._region(lay, "x_perm", torch.bfloat16, (pairs, self.d)), self.experts[0], offsets, h, True)
        self._product(h, self.experts[1], offsets, self.y_perm, False)
        self.ctx.combine_routed(gates, pairs, y, self.workspace, self.stream)

    def router_gradient(self, logits, dy, d_loss, mask=None):
        """Gradient of the last forward call's logits (the same logits and mask are given again) from that of y (bf16 [T, d_model]) and of
        the balance loss (fp32 [1]).  A gate's is the product of dy with its expert's output."""
        T = self.tokens
        self._need(logits, "logits", (T, self.E))
        self._need(dy, "dy", (T, self.d), (torch.bfloat16, torch.float32, torch.float16, torch.float64))
        out = torch.empty_like(logits)
        if T:
            with self._on_stream():
                rows = self.y_perm[self.inv.long()].view(T, self.k, self.d)
                d_gates = (rows.float() * dy.float()[:, None, :]).sum(2)
                route_backward(logits, self.ids[:T], self.counts, out, self.stream, d_gates=d_gates, d_loss=d_loss, mask=mask,
                               normalize=self.normalize)
        return out

    def close(self):
        self.ctx.close()
