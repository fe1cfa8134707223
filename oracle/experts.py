"""Plain definitions, in 64 bits, of the way of tokens to their experts and back and of the experts' products (test infrastructure only)."""
from __future__ import annotations

import math

import torch


def sort(ids, gates, E):
    """(offsets [E+1], places [T,k]) of ids [T,k]: pairs with an id in [0,E) and a gate that is not 0, by expert and then in their order."""
    places, offsets, at = torch.full(ids.shape, -1, dtype=torch.int32), [0], 0
    for e in range(E):
        for t, j in (ids == e).nonzero().tolist():
            if gates is None or float(gates[t, j]) != 0:
                places[t, j] = at
                at += 1
        offsets.append(at)
    return torch.tensor(offsets, dtype=torch.int32), places


def rows(x, places, out):
    out = out.double().clone()
    for t, j in (places >= 0).nonzero().tolist():
        out[places[t, j]] = x[t].double()
    return out


def combine(rows, places, gates, residual, d):
    y = torch.zeros((places.shape[0], d), dtype=torch.float64) if residual is None else residual.double().clone()
    for t, j in (places >= 0).nonzero().tolist():
        y[t] += (1.0 if gates is None else float(gates[t, j])) * rows[places[t, j]].double()
    return y


def combine_backward(dy, rows, places, gates, d_rows):
    """(d_rows, d_gates)"""
    d_rows, d_gates = d_rows.double().clone(), torch.zeros(places.shape, dtype=torch.float64)
    for t, j in (places >= 0).nonzero().tolist():
        at = int(places[t, j])
        d_rows[at] = (1.0 if gates is None else float(gates[t, j])) * dy[t].double()
        if rows is not None:
            d_gates[t, j] = (dy[t].double() * rows[at].double()).sum()
    return d_rows, d_gates


def argument(v, act):
    """What the sigmoid of v * sigmoid(.) is taken of."""
    return v if act == "silu" else 2 * math.sqrt(2 / math.pi) * (v + 0.044715 * v ** 3)


def activation(v, act):
    if act == "none":
        return v
    if act == "relu":
        return torch.where(v > 0, v, v * 0)
    return v * torch.sigmoid(argument(v, act))


def slope(v, act):
    if act == "none":
        return torch.ones_like(v)
    if act == "relu":
        return (v > 0).double()
    s = torch.sigmoid(argument(v, act))
    du = torch.ones_like(v) if act == "silu" else 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * v ** 2)
    return s + v * s * torch.sigmoid(-argument(v, act)) * du


def product(x, w, bounds):
    """(v, sum of magnitudes): x [M,K], w [groups,N,K]; rows of no group are 0."""
    v = torch.zeros((x.shape[0], w.shape[1]), dtype=torch.float64)
    size = v.clone()
    for g, (a, b) in enumerate(zip(bounds[:-1], bounds[1:])):
        if b > a:
            v[a:b] = x[a:b].double() @ w[g].double().t()
            size[a:b] = x[a:b].double().abs() @ w[g].double().abs().t()
    return v, size


def input_gradient(dy, w, bounds):
    return product(dy, w.transpose(1, 2), bounds)


def weights_gradient(dy, x, bounds):
    """(dw, its sum of magnitudes, d_bias, its sum of magnitudes)"""
    dy, x = dy.double(), x.double()
    parts = [(dy[a:b], x[a:b]) if b > a else (dy[:0], x[:0]) for a, b in zip(bounds[:-1], bounds[1:])]
    return (torch.stack([p.t() @ q for p, q in parts]), torch.stack([p.abs().t() @ q.abs() for p, q in parts]),
            torch.stack([p.sum(0) for p, _ in parts]), torch.stack([p.abs().sum(0) for p, _ in parts]))
