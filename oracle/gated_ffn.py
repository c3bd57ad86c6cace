"""The gated feed-forward block and its gradients from their formulas, in 64 bits (torch on any device), with a bound
for each output on how far a 32-bit computation may be from it.

    h = D act(x Wg^T) (x Wu^T);  e = D dh;  dU = e act(G);  dG = e U act'(G)
    dx = dG Wg + dU Wu;  dWg = dG^T x;  dWu = dU^T x

Bounds.  A sum of n products in 32 bits, in any order, whose additions may round to nearest or truncate, is off by at
most (n + 2) 2^-23 times the sum of the products' magnitudes.  G and U are such sums; what follows is propagated to
first order with the activations' largest slopes, plus a few units of 2^-22 for the activation itself; a result
rounded to a type of p bits adds 2^-p of its magnitude (and half the smallest step of a 16-bit float).
"""
from __future__ import annotations

import math
from dataclasses import dataclass

import torch

from . import dropout_numpy

UNIT = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8}
TINY = {torch.float32: 2.0 ** -149, torch.float16: 2.0 ** -25, torch.bfloat16: 2.0 ** -134}
# largest slope of act and of act' (silu: 1.0999 and 0.5; gelu: 1.1289 and 0.798; relu's own steps are handled apart)
SLOPE = {"relu": 1.0, "silu": 1.1, "gelu": 1.13}
CURVE = {"relu": 0.0, "silu": 0.5, "gelu": 0.8}


def act(g: torch.Tensor, name: str):
    """act(g) and act'(g)."""
    if name == "relu":
        on = (g > 0) | torch.isnan(g)
        return torch.where(on, g, torch.zeros_like(g)), on.to(g.dtype)
    if name == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * torch.sigmoid(-g))
    phi = torch.special.ndtr(g)
    return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def keep_mask(m, f, p, seed, sequence, device):
    if dropout_numpy.threshold(p) == 0:
        return torch.ones(m, f, dtype=torch.bool, device=device)
    return torch.from_numpy(dropout_numpy.keep_mask(m, f, p, seed, sequence)).to(device)


@dataclass
class Result:
    """value and bound of each output"""
    value: dict
    bound: dict


def _sum_bound(n):
    return (n + 2) * 2.0 ** -23


def _gate(x, wg, wu):
    g, u = x @ wg.t(), x @ wu.t()
    s = _sum_bound(x.shape[1])
    return g, u, s * (x.abs() @ wg.abs().t()), s * (x.abs() @ wu.abs().t())


def forward(x, wg, wu, name, p=0.0, seed=0, sequence=0) -> Result:
    dtype = x.dtype
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u, eg, eu = _gate(x, wg, wu)
    a, _ = act(g, name)
    keep = keep_mask(x.shape[0], wg.shape[0], p, seed, sequence, x.device)
    scale = dropout_numpy.scale(p)
    h = torch.where(keep, a * u * scale, torch.zeros_like(a))
    ea = SLOPE[name] * eg + 2.0 ** -20 * a.abs() + 2.0 ** -22 * g.abs() * (g.abs() < 20)
    err = scale * (ea * u.abs() + a.abs() * eu + ea * eu) + 2.0 ** -22 * h.abs()
    return Result({"h": h}, {"h": torch.where(keep, err * (1 + UNIT[dtype]) + UNIT[dtype] * h.abs() + TINY[dtype], torch.zeros_like(h))})


def backward(x, wg, wu, dh, name, p=0.0, seed=0, sequence=0) -> Result:
    dtype = x.dtype
    unit, tiny = UNIT[dtype], TINY[dtype]
    x, wg, wu, dh = x.double(), wg.double(), wu.double(), dh.double()
    g, u, eg, eu = _gate(x, wg, wu)
    a, slope = act(g, name)
    keep = keep_mask(x.shape[0], wg.shape[0], p, seed, sequence, x.device)
    e = torch.where(keep, dh * dropout_numpy.scale(p), torch.zeros_like(dh))
    du, dg = e * a, e * u * slope
    ea = SLOPE[name] * eg + 2.0 ** -20 * a.abs() + 2.0 ** -22 * g.abs() * (g.abs() < 20)
    es = CURVE[name] * eg + 2.0 ** -20
    if name == "relu":      # the slope itself hangs on the sign of G where rounding can turn it
        es = (g.abs() <= eg).double()
    edu = e.abs() * ea + 2.0 ** -22 * du.abs()
    edg = e.abs() * (u.abs() * es + slope.abs() * eu + eu * es) + 2.0 ** -22 * dg.abs()
    if dtype != torch.float32:      # rounded to the element type between the products
        edu = edu * (1 + unit) + unit * du.abs() + tiny
        edg = edg * (1 + unit) + unit * dg.abs() + tiny
    value = {"dx": dg @ wg + du @ wu, "dwg": dg.t() @ x, "dwu": du.t() @ x}
    sf, sm = _sum_bound(2 * wg.shape[0]), _sum_bound(x.shape[0])
    bound = {
        "dx": edg @ wg.abs() + edu @ wu.abs() + sf * ((dg.abs() + edg) @ wg.abs() + (du.abs() + edu) @ wu.abs()),
        "dwg": edg.t() @ x.abs() + sm * ((dg.abs() + edg).t() @ x.abs()),
        "dwu": edu.t() @ x.abs() + sm * ((du.abs() + edu).t() @ x.abs()),
    }
    return Result(value, {n: b * (1 + unit) + unit * value[n].abs() + tiny for n, b in bound.items()})
