"""The parts of a block on histories (layer norm, causal attention, gated feed-forward) in 64 bits, on the CPU, each with a bound on the error of fp32
arithmetic (and of bf16 operands and outputs where the tensors are bf16), element by element, from the standard model of rounding: a sum in which every term goes through
at most d additions is off by at most (d + 1) u times the sum of the terms' magnitudes."""
from __future__ import annotations

import math

import torch

from tests.seq_ref import U, UB, out_round


def _depth(channels):
    """Additions that a term of a row's sum goes through: a lane's own (up to 64, or every 256th of a wide row), then the lanes' and waves'."""
    return 80 + channels // 256


def norm(x, residual, weight, bias, eps):
    """(y, s, stats, bounds of the three)."""
    dtype, C = x.dtype, x.shape[1]
    s = x.double() + (0 if residual is None else residual.double())
    es = torch.zeros_like(s) if residual is None else U * s.abs()
    d = _depth(C)
    mean = s.mean(1, keepdim=True)
    em = (d + 3) * U * s.abs().mean(1, keepdim=True) + es.mean(1, keepdim=True)
    x0 = s - mean
    ex = es + em + U * x0.abs()
    var = x0.square().mean(1, keepdim=True)
    ev = 2 * (x0.abs() * ex).mean(1, keepdim=True) + ex.square().mean(1, keepdim=True) + (d + 4) * U * var
    rstd = (var + eps).rsqrt()
    rel = 0.5 * ev / (var + eps) * 1.1 + 8 * U     # (eps is itself an fp32 number; a sum, a root and a quotient of at most two ulps each)
    h = x0 * rstd
    eh = ex * rstd * (1 + rel) + h.abs() * (rel + U)
    w, b = (torch.ones(C, dtype=torch.float64) if weight is None else weight.double()), (torch.zeros(C, dtype=torch.float64) if bias is None else bias.double())
    y = h * w + b
    ey = w.abs() * eh + 2 * U * ((h * w).abs() + b.abs())
    slack = UB * 1.01 if dtype == torch.bfloat16 else U
    stats, est = torch.cat([mean, rstd], 1), torch.cat([em, rel * rstd], 1)
    return y, s, stats, ey + slack * (y.abs() + ey), es + slack * (s.abs() + es), est + U * stats.abs()


def norm_grad(dy, s, stats, weight, dsum):
    """(ds, dweight, dbias, bounds of the three), from s and stats as given."""
    dtype, (n, C) = s.dtype, s.shape
    mean, rstd = stats.double().split(1, 1)
    h, y = (s.double() - mean) * rstd, dy.double()
    g = y * (1.0 if weight is None else weight.double())
    d = _depth(C)
    s0, s1 = g.mean(1, keepdim=True), (g * h).mean(1, keepdim=True)
    e = torch.zeros_like(g) if dsum is None else dsum.double()
    ds = rstd * (g - s0 - h * s1) + e
    err = rstd * ((d + 8) * U * g.abs().mean(1, keepdim=True) + h.abs() * (d + 10) * U * (g * h).abs().mean(1, keepdim=True) + 8 * U * (g.abs() + s0.abs() + (h * s1).abs()))
    err = err + 2 * U * (ds.abs() + e.abs())
    dw, db = (y * h).sum(0), y.sum(0)
    return (ds, dw, db, err + out_round(ds, dtype) * 1.01, (n + 16) * U * (y * h).abs().sum(0) + 1e-37, (n + 16) * U * y.abs().sum(0) + 1e-37)
