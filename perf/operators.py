"""Operator cases: experts held in microscaled 4 bits, and the router whose balance is trained.

  quantize   rows of bf16 or fp32 values to MXFP4: 4-bit values (1 sign, 2 exponent, 1 mantissa bit), one power of two
             for each 32 of them (``mx_quantize``); comes back as the values that the codes stand for
  product    tokens in expert order times the experts' MXFP4 weights (``mx_gemm``); the tokens are bf16, or are
             quantised within the pass and multiplied as MXFP4 (``x4``)
  route      router logits to experts, gates, tokens per expert and the balance loss (``route``)
  route_grad the gradient of the logits from those of the gates and the loss (``route_backward``)

Shapes are those of ``workloads`` and ``bench.py``: layers of 768 x 3072 and 1024 x 4096, 8 to 256 experts with Zipf
popularity, batches from one token to 32768.  Activations N(0, 1), hidden values their positive part, expert weights
N(0, 0.02).  A state holds the weights' codes twice: row by row, and in the order that the matrix product takes.
"""
from __future__ import annotations

import math

import torch

own = False

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)  # what the codes 0..7 stand for; code + 8 is the negative

# Most work of a drawn case: that of the largest case of its kind below.
MOST_WEIGHTS, MOST_FLOPS = 128 * 4096 * 1024, 2.0 * 32768 * 4096 * 1024
MOST_VALUES, MOST_LOGITS = 64 * 4096 * 1024, 262144 * 128


def _quantize(name, rows, cols, dtype, tiles):
    return {"name": name, "kind": "quantize", "rows": rows, "cols": cols, "dtype": dtype, "tiles": tiles}


def _product(name, E, K, N, M, zipf, x4=False, relu=False, y32=False):
    return {"name": name, "kind": "product", "E": E, "K": K, "N": N, "M": M, "zipf": zipf, "x4": x4, "relu": relu, "y32": y32}


def _route(name, kind, T, E, k, dtype, normalize=False, mask=False):
    return {"name": name, "kind": kind, "T": T, "E": E, "k": k, "dtype": dtype, "normalize": normalize, "mask": mask}


def listed():
    return [
        # One token's activations: the smallest call, all latency.
        _quantize("quantize-token", 1, 1024, "bf16", False),
        # The first matrices of 64 experts of the larger model, from fp32 master weights, when a model is loaded.
        _quantize("quantize-experts", 64 * 4096, 1024, "fp32", True),
        # Decoding, one token: one expert's second matrix is read.
        _product("product-1-token", 128, 4096, 1024, 1, 1.0, y32=True),
        # One sentence through Switch-base-128's first matrices: two or three tokens for each of 50 experts.
        _product("product-128-tokens", 128, 768, 3072, 128, 1.0, relu=True),
        # An odd, middling batch through the second matrices of 64 experts.
        _product("product-1111-tokens", 64, 3072, 768, 1111, 1.2),
        # The benchmark's batch, first matrices.
        _product("product-16384-tokens", 128, 768, 3072, 16384, 1.0, relu=True),
        # Tokens in 4 bits too: a few paragraphs with three experts each, first matrices of the larger model.
        _product("product-4bit-999", 64, 1024, 4096, 999, 0.8, x4=True, relu=True),
        # The larger model's largest batch, second matrices, tokens in 4 bits.
        _product("product-4bit-32768", 128, 4096, 1024, 32768, 1.2, x4=True),
        # A sentence's router.
        _route("route-128-tokens", "route", 128, 128, 1, "bf16"),
        # A large batch, three of 256 experts with gates that sum to one, padded tokens masked.
        _route("route-32768-tokens", "route", 32768, 256, 3, "fp32", normalize=True, mask=True),
        # Gradients: an odd batch in bf16 ...
        _route("route-grad-1111", "route_grad", 1111, 64, 2, "bf16", normalize=True, mask=True),
        # ... and a training batch of 64 sequences of 4096 tokens.
        _route("route-grad-262144", "route_grad", 262144, 128, 1, "fp32"),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(("quantize", "product", "product", "route", "route_grad"))
    if kind == "quantize":
        cols = 32 * _log_int(rng, 2, 128)
        rows = _log_int(rng, 1, min(262144, MOST_VALUES // cols))
        return {"kind": kind, "rows": rows, "cols": cols, "dtype": rng.choice(("bf16", "fp32")), "tiles": rng.random() < 0.5}
    if kind == "product":
        K, N = 32 * _log_int(rng, 8, 128), _log_int(rng, 64, 4096)
        E = _log_int(rng, 1, min(256, MOST_WEIGHTS // (K * N)))
        M = _log_int(rng, 1, min(32768, int(MOST_FLOPS / (2.0 * K * N))))
        return {"kind": kind, "E": E, "K": K, "N": N, "M": M, "zipf": rng.choice((0.0, 0.8, 1.0, 1.2)),
                "x4": rng.random() < 0.4, "relu": rng.random() < 0.5, "y32": rng.random() < 0.2}
    E = _log_int(rng, 8, 256)
    T = _log_int(rng, 1, min(262144, MOST_LOGITS // E))
    return {"kind": kind, "T": T, "E": E, "k": min(E, rng.choice((1, 1, 2, 3, 8))), "dtype": rng.choice(("bf16", "fp32")),
            "normalize": rng.random() < 0.5, "mask": rng.random() < 0.5}


# ---- inputs -------------------------------------------------------------------------------------
def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _encode(w):
    """MXFP4 codes uint8 [rows, cols / 2] and scales uint8 [rows, cols / 32] of fp32 rows."""
    rows, cols = w.shape
    b = w.view(rows, cols // 32, 32)
    e = torch.frexp(b.abs().amax(2)).exponent - 3          # floor(log2(largest)) - 2
    v = torch.ldexp(b, -e[:, :, None]).view(rows, cols)
    a = v.abs()
    # the code of a magnitude counts the midpoints below it; a value on a midpoint takes the even code
    code = torch.zeros_like(a, dtype=torch.uint8)
    for i, mid in enumerate((0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0)):
        code += (a >= mid) if i % 2 else (a > mid)
    code |= (v < 0).to(torch.uint8) << 3
    return code[:, 0::2] | code[:, 1::2] << 4, (e + 127).clamp(0, 254).to(torch.uint8)


def _in_tiles(codes, scales, E, N, K):
    """The two in the order of the matrix product: stripes of 32 rows, 64 columns (codes) or 256 (scales) at a time."""
    n, k = -(-N // 32) * 32, -(-K // 64) * 64
    c = torch.zeros((E, n, k // 2), dtype=torch.uint8, device="cuda")
    c[:, :N, : K // 2] = codes.view(E, N, K // 2)
    c = c.view(E, n // 32, 32, k // 64, 2, 16).permute(0, 1, 3, 4, 2, 5).contiguous()
    k = -(-K // 256) * 256
    s = torch.full((E, n, k // 32), 127, dtype=torch.uint8, device="cuda")
    s[:, :N, : K // 32] = scales.view(E, N, K // 32)
    s = s.view(E, n // 32, 32, k // 256, 4, 2).permute(0, 1, 3, 5, 2, 4).contiguous()
    return c.view(-1), s.view(-1)


def _ids(case, g, E, M):
    """Experts of M tokens, ascending: popularity rank r with probability as r ** -zipf."""
    p = torch.arange(1, E + 1, device="cuda", dtype=torch.float64) ** -float(case["zipf"])
    cdf = torch.cumsum(p / p.sum(), 0)
    rank = torch.searchsorted(cdf, torch.rand(M, generator=g, device="cuda", dtype=torch.float64)).clamp_(max=E - 1)
    return torch.randperm(E, generator=g, device="cuda")[rank]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed) * 7919 + 17)
    state = {"case": case, "stream": torch.cuda.current_stream()}

    def normal(*shape, dtype=torch.float32):
        return torch.randn(shape, generator=g, device="cuda", dtype=dtype)

    if case["kind"] == "quantize":
        rows, cols = case["rows"], case["cols"]
        x = normal(rows, cols, dtype=_dtype(case))
        state["x"] = x * 0.02 if case["tiles"] else x
        r, k = (-(-rows // 32) * 32, -(-cols // 64) * 64) if case["tiles"] else (rows, cols)
        state["codes"] = torch.empty(r * k // 2, dtype=torch.uint8, device="cuda")
        state["scales"] = torch.empty(r * (-(-cols // 256) * 8), dtype=torch.uint8, device="cuda")
        state["values"] = torch.empty((rows, cols), dtype=torch.bfloat16, device="cuda")
    elif case["kind"] == "product":
        E, K, N, M = (case[n] for n in "EKNM")
        parts = [_encode((normal(n, K) * 0.02).bfloat16().float()) for n in _pieces(E * N, K)]
        codes, scales = (torch.cat([p[i] for p in parts]) for i in (0, 1))
        state["codes"], state["scales"] = codes.view(E, N, K // 2), scales.view(E, N, K // 32)
        state["tile_codes"], state["tile_scales"] = _in_tiles(codes, scales, E, N, K)
        grid = torch.tensor(GRID + tuple(-v for v in GRID), device="cuda")
        state["pairs"] = torch.stack((grid.repeat(16), grid.repeat_interleave(16)), 1)   # the two values of a byte
        x = normal(M, K, dtype=torch.bfloat16)
        state["x"] = x if case["relu"] else x.clamp_min(0)   # a second matrix's tokens are hidden values
        counts = torch.bincount(_ids(case, g, E, M), minlength=E)
        state["offsets"] = torch.zeros(E + 1, dtype=torch.int32, device="cuda")
        state["offsets"][1:] = torch.cumsum(counts, 0)
        state["bounds"] = state["offsets"].tolist()          # as a plan has them on the host
        state["y"] = torch.empty((M, N), dtype=torch.float32 if case["y32"] else torch.bfloat16, device="cuda")
        state["x_codes"] = torch.empty((M, K // 2), dtype=torch.uint8, device="cuda")
        state["x_scales"] = torch.empty((M, -(-K // 256) * 8), dtype=torch.uint8, device="cuda")
    else:
        T, E, k = case["T"], case["E"], case["k"]
        liked = torch.log(torch.arange(1, E + 1, device="cuda") ** -0.8)[torch.randperm(E, generator=g, device="cuda")]
        state["logits"] = (normal(T, E) * 1.5 + liked).to(_dtype(case))
        state["mask"] = (torch.rand(T, generator=g, device="cuda") < 0.9) if case["mask"] else None
        state["ids"] = torch.empty((T, k), dtype=torch.int32, device="cuda")
        state["gates"] = torch.empty((T, k), device="cuda")
        state["counts"] = torch.empty(E, dtype=torch.int32, device="cuda")
        state["loss"] = torch.empty((), device="cuda")
        state["workspace"] = torch.empty(1 << 20, dtype=torch.uint8, device="cuda")
        if case["kind"] == "route_grad":                     # what the forward pass has left
            ids = torch.sort(state["logits"], dim=1, descending=True, stable=True).indices[:, :k]
            state["ids"].copy_(ids)
            valid = state["mask"] if case["mask"] else torch.ones(T, dtype=torch.bool, device="cuda")
            state["counts"].copy_(torch.bincount(ids[valid].reshape(-1), minlength=E))
            state["d_gates"] = normal(T, k) / T
            state["d_loss"] = torch.full((), 0.01, device="cuda")
            state["d_logits"] = torch.empty_like(state["logits"])
    torch.cuda.synchronize()
    return state


def _pieces(rows, cols):
    """Row counts of pieces of at most 2^26 values."""
    step = max(1, (1 << 26) // cols)
    return [min(step, rows - r) for r in range(0, rows, step)]


# ---- one pass -----------------------------------------------------------------------------------
def run(state):
    case = state["case"]
    return (_run_own if own else _run_plain)(state, case, case["kind"])


def _run_own(state, case, kind):
    import paper_2310_18859_amd as sm
    s = state["stream"]
    if kind == "quantize":
        sm.mx_quantize(state["x"], state["codes"], state["scales"], s, layout=sm.MX_TILES if case["tiles"] else sm.MX_ROWS,
                       values=state["values"])
        return state["values"]
    if kind == "product":
        x, x_scales = state["x"], None
        if case["x4"]:
            sm.mx_quantize(x, state["x_codes"], state["x_scales"], s)
            x, x_scales = state["x_codes"], state["x_scales"]
        sm.mx_gemm(x, x_scales, state["tile_codes"], state["tile_scales"], state["offsets"], state["y"], s, relu=case["relu"])
        return state["y"]
    if kind == "route":
        sm.route(state["logits"], state["ids"], state["gates"], state["counts"], state["loss"], state["workspace"], s,
                 mask=state["mask"], normalize=case["normalize"])
        return {n: state[n] for n in ("ids", "gates", "counts", "loss")}
    sm.route_backward(state["logits"], state["ids"], state["counts"], state["d_logits"], s, d_gates=state["d_gates"],
                      d_loss=state["d_loss"], mask=state["mask"], normalize=case["normalize"])
    return state["d_logits"]


def _nearest(x):
    """x rounded to MXFP4 in blocks of 32 along its rows, as fp32 values."""
    rows, cols = x.shape
    b = x.float().view(rows, cols // 32, 32)
    scale = torch.frexp(b.abs().amax(2, keepdim=True)).exponent.clamp(min=-124) - 3
    v = torch.ldexp(b, -scale)
    step = torch.frexp(v).exponent.clamp(min=1) - 2          # one mantissa bit; below 1 the step stays 1/2
    v = torch.ldexp(torch.round(torch.ldexp(v, -step)), step).clamp(-6, 6)
    return torch.ldexp(v, scale).view(rows, cols)


def _decode(codes, scales, pairs):
    """fp32 values [N, K] of one expert's codes and scales."""
    v = pairs[codes.int()].view(*scales.shape, 32)
    return (v * torch.exp2(scales.float() - 127)[:, :, None]).view(codes.shape[0], -1)


def _softmax(logits):
    e = torch.exp(logits - logits.amax(1, keepdim=True))
    return e / e.sum(1, keepdim=True)


def _run_plain(state, case, kind):
    if kind == "quantize":
        return _nearest(state["x"]).bfloat16()
    if kind == "product":
        x = _nearest(state["x"]) if case["x4"] else state["x"].float()
        at = state["bounds"]
        y = torch.empty((case["M"], case["N"]), device="cuda")
        for e in range(case["E"]):                           # a product for each expert that has tokens
            if at[e + 1] > at[e]:
                torch.mm(x[at[e]:at[e + 1]], _decode(state["codes"][e], state["scales"][e], state["pairs"]).t(), out=y[at[e]:at[e + 1]])
        if case["relu"]:
            y = y.clamp_min_(0)
        return y if case["y32"] else y.bfloat16()
    E, k = case["E"], case["k"]
    logits = state["logits"].float()
    p = _softmax(logits)
    valid = state["mask"].float()[:, None] if case["mask"] else torch.ones_like(p[:, :1])
    n = valid.sum().clamp_min(1)
    if kind == "route":
        ids = torch.sort(logits, dim=1, descending=True, stable=True).indices[:, :k]
        gates = torch.gather(p, 1, ids)
        if case["normalize"]:
            gates = gates / gates.sum(1, keepdim=True)
        ones = valid.int().expand(-1, k).reshape(-1)
        counts = torch.zeros(E, dtype=torch.int32, device="cuda").scatter_add_(0, ids.reshape(-1), ones)
        loss = E * (counts / (n * k) * (p * valid).sum(0) / n).sum()
        return {"ids": ids.int(), "gates": gates * valid, "counts": counts, "loss": loss}
    dp = (state["d_loss"] * E / n * (state["counts"] / (n * k))).expand_as(p).clone()
    ids, dg = state["ids"].long(), state["d_gates"]
    if case["normalize"]:
        gates = torch.gather(p, 1, ids)
        total = gates.sum(1, keepdim=True)
        dg = (dg - (dg * gates).sum(1, keepdim=True) / total) / total
    dp.scatter_add_(1, ids, dg)
    return (valid * p * (dp - (p * dp).sum(1, keepdim=True))).to(_dtype(case))


# ---- the same from the definitions, in 64 bits ---------------------------------------------------
def _exact_mx(x):
    """x [rows, cols] rounded to MXFP4: of the eight magnitudes the nearest one, of two as near the one with the even code."""
    rows, cols = x.shape
    b = x.double().view(rows, cols // 32, 32)
    unit = 2.0 ** (torch.floor(torch.log2(b.abs().amax(2, keepdim=True).clamp_min(2.0 ** -125))) - 2)
    a = b.abs() / unit
    at = torch.tensor(GRID, device="cuda", dtype=torch.float64)
    hi = torch.searchsorted(at, a.contiguous()).clamp_(1, 7)
    down, up = a - at[hi - 1], at[hi] - a
    pick = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    return (torch.sign(b) * at[pick] * unit).view(rows, cols)


def _exact_weights(codes, scales):
    low, high = codes % 16, codes // 16
    nib = torch.stack((low, high), -1).flatten(-2)
    exp, man = (nib // 2 % 4).double(), (nib % 2).double()
    mag = torch.where(exp > 0, (1 + man / 2) * 2.0 ** (exp - 1), man / 2)
    return torch.where(nib > 7, -mag, mag) * (2.0 ** (scales.double() - 127)).repeat_interleave(32, -1)


def exact(case, seed):
    state = prepare(case, seed)
    if case["kind"] == "quantize":
        x, out = state["x"], torch.empty(state["x"].shape, device="cuda", dtype=torch.float64)
        at = 0
        for n in _pieces(*x.shape):
            out[at:at + n] = _exact_mx(x[at:at + n])
            at += n
        return out
    if case["kind"] == "product":
        x = _exact_mx(state["x"]) if case["x4"] else state["x"].double()
        y = torch.zeros((case["M"], case["N"]), device="cuda", dtype=torch.float64)
        at = state["bounds"]
        for e in range(case["E"]):
            a, b = at[e], at[e + 1]
            if b > a:
                y[a:b] = x[a:b] @ _exact_weights(state["codes"][e], state["scales"][e]).T.contiguous()
        return torch.relu(y) if case["relu"] else y
    E, k, T = case["E"], case["k"], case["T"]
    z = state["logits"].double()
    p = torch.exp(z - torch.logsumexp(z, 1, keepdim=True))
    valid = state["mask"].double() if case["mask"] else torch.ones(T, device="cuda", dtype=torch.float64)
    n = max(1.0, float(valid.sum()))
    if case["kind"] == "route":
        work, ids = z.clone(), []
        for _ in range(k):                                   # the largest, the lowest of equal ones, and again without it
            best = (work == work.amax(1, keepdim=True)).double().argmax(1)
            ids.append(best)
            work[torch.arange(T, device="cuda"), best] = -math.inf
        ids = torch.stack(ids, 1)
        gates = torch.gather(p, 1, ids)
        counts = torch.bincount(ids[valid > 0].reshape(-1), minlength=E)
        loss = E * ((counts.double() / (n * k)) * ((valid[:, None] * p).sum(0) / n)).sum()
        return {"ids": ids.int(), "gates": (gates / gates.sum(1, keepdim=True) if case["normalize"] else gates) * valid[:, None],
                "counts": counts.int(), "loss": loss}
    ids, dg = state["ids"].long(), state["d_gates"].double()
    picked = torch.gather(p, 1, ids)
    # d gate_j / d z_i = gate_j (i == j) - gate_j p_i, and with p_i only among the chosen where gates sum to one
    out = torch.zeros_like(p)
    gates = picked / picked.sum(1, keepdim=True) if case["normalize"] else picked
    mean = (dg * gates).sum(1, keepdim=True)
    if case["normalize"]:
        out.scatter_add_(1, ids, gates * (dg - mean))
    else:
        out.scatter_add_(1, ids, gates * dg)
        out -= mean * p
    pull = E * state["counts"].double() / (n * k) / n * float(state["d_loss"])
    out += p * (pull - (p * pull).sum(1, keepdim=True))
    return out * valid[:, None]


# ---- what a pass cannot do without --------------------------------------------------------------
def work(case):
    if case["kind"] == "quantize":
        n = float(case["rows"]) * case["cols"]
        # values in; 4 bits each and a byte per 32, and the rounded values as bf16, out
        return {"bytes": n * ((2 if case["dtype"] == "bf16" else 4) + 0.5 + 1 / 32 + 2), "flops": n * 4}
    if case["kind"] == "product":
        E, K, N, M = (case[n] for n in "EKNM")
        p = [r ** -float(case["zipf"]) for r in range(1, E + 1)]
        active = sum(1.0 - (1.0 - v / sum(p)) ** M for v in p)
        return {"bytes": active * K * N * (0.5 + 1 / 32) + M * (2.0 * K + (4.0 if case["y32"] else 2.0) * N) + 4.0 * (E + 1),
                "flops": 2.0 * M * K * N}
    T, E, k, size = case["T"], case["E"], case["k"], 2 if case["dtype"] == "bf16" else 4
    masks = T if case["mask"] else 0
    if case["kind"] == "route":
        return {"bytes": T * (float(size) * E + 8 * k) + masks + 4 * E + 4, "flops": 4.0 * T * E}
    return {"bytes": T * (2.0 * size * E + 8 * k) + masks + 4 * E + 4, "flops": 6.0 * T * E}
