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


def _causal_pairs(q, k, q_off, k_start, k_len, mask):
    """Per sequence and head: the rows, the keys that count, which of them a row does not see, and which rows see any."""
    H, G = q.shape[1], k.shape[1]
    for s in range(len(q_off) - 1):
        nq, n = q_off[s + 1] - q_off[s], torch.arange(k_len[s])
        if mask is not None:
            n = n[mask[k_start[s] + n] != 0]
        if not nq or not len(n):
            continue
        hidden = n[None] > torch.arange(nq)[:, None] + (k_len[s] - nq)
        for h in range(H):
            yield slice(q_off[s], q_off[s + 1]), k_start[s] + n, hidden, h, h // (H // G)


def _scores(q, k, scale, hidden):
    """Scores and the error of their exponential: the product's, the rounding of scale * log2(e) and of its product with the score, and the exponential's own."""
    s = q @ k.T * scale
    es = U * ((q.shape[1] + 4) * scale * (q.abs() @ k.abs().T) + 4 * s.abs() + 8)
    return s.masked_fill(hidden, -math.inf), es.masked_fill(hidden, 0.0)


def attend(q, k, v, q_off, k_start, k_len, scale, mask):
    """(o, lse, bounds of both) in causal order: query i of nq sees the keys up to i + nk - nq."""
    dtype = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    o, eo = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -math.inf, dtype=torch.float64)
    el = torch.zeros(q.shape[:2], dtype=torch.float64)
    for rows, keys, hidden, h, g in _causal_pairs(q, k, q_off, k_start, k_len, mask):
        s, es = _scores(q[rows, h], k[keys, g], scale, hidden)
        some = ~hidden.all(1)
        l = torch.logsumexp(s, 1)
        p = torch.exp(s - torch.where(some, l, 0.0)[:, None])
        mean = (p * es).sum(1, keepdim=True)
        # (each rescaling to a new maximum costs an exponential and a product: at most one per 32 keys and one per piece)
        w = p * (es + mean + (3 * len(keys) + 64) * U + (UB if dtype == torch.bfloat16 else 0.0))
        o[rows, h], lse[rows, h] = p @ v[keys, g], l
        eo[rows, h] = w @ v[keys, g].abs() + out_round(o[rows, h], dtype)
        top = s.masked_fill(hidden, 0.0).abs().amax(1)
        el[rows, h] = mean[:, 0] + (len(keys) + 64) * U + 4 * U * torch.where(some, l, 0.0).abs() + 4 * U * top
    return o, lse, eo, el


def attend_grad(dout, q, k, v, o, lse, q_off, k_start, k_len, scale, mask):
    """(dq, dk, dv, bounds of the three), from o and lse as given."""
    dtype = q.dtype
    ub = UB if dtype == torch.bfloat16 else 0.0
    dout, q, k, v, o, lse = (t.double() for t in (dout, q, k, v, o, lse))
    dq, dk, dv, eq, ek, ev = (torch.zeros_like(t) for t in (q, k, v, q, k, v))
    for rows, keys, hidden, h, g in _causal_pairs(q, k, q_off, k_start, k_len, mask):
        n, m, D = len(keys), rows.stop - rows.start, q.shape[2]
        some = ~hidden.all(1, keepdim=True)
        clean = lambda t: torch.where(some, t[rows, h], 0.0)  # noqa: E731
        qr, do, orow, kr, vr = clean(q), clean(dout), clean(o), k[keys, g], v[keys, g]
        l = torch.where(some[:, 0], lse[rows, h], 0.0)[:, None]
        s, es = _scores(qr, kr, scale, hidden)
        p = torch.exp(s - l)
        es = es + 4 * U * l.abs()
        dp, delta = do @ vr.T, (do * orow).sum(1, keepdim=True)
        ds = p * (dp - delta)
        eds = ds.abs() * (es + 4 * U + ub) + p * U * ((D + 4) * (do.abs() @ vr.abs().T) + (D + 4) * (do * orow).abs().sum(1, keepdim=True) + dp.abs() + delta.abs())
        dq[rows, h] = scale * ds @ kr
        eq[rows, h] = scale * (eds @ kr.abs() + (n + 8) * U * (ds.abs() @ kr.abs()))
        dk[keys, g] += scale * ds.T @ qr
        ek[keys, g] += scale * (eds.T @ qr.abs() + (m * 4 + 8) * U * (ds.abs().T @ qr.abs()))
        dv[keys, g] += p.T @ do
        ev[keys, g] += (p * (es + ub)).T @ do.abs() + (m * 4 + 8) * U * (p.T @ do.abs())
    return dq, dk, dv, eq + out_round(dq, dtype), ek + out_round(dk, dtype), ev + out_round(dv, dtype)


# ---------------------------------------------------------------------------------------------- gated feed-forward
# A sigmoid: its exponent is rounded (|x| log2(e), 1.5 |x| u), the exponential, a sum and a reciprocal are good to two ulps each: (1.5 |x| + 10) u of the value.
# The normal distribution's function by a formula that is off by 0.75e-7, its sums and products by another 8 u; all of it times x.
PHI = 0.75e-7 + 8 * U
# What lies below the smallest normal number, 2^-126, may come out as zero (a reciprocal of more than 2^126, an exponential): an absolute error of that in a sigmoid,
# a tail or a density, which a product with g carries on (sigmoid(-88) = 6e-39, 88 times that is 5e-37).
UNDER = 2.0 ** -125


def act(name, g):
    """(act(g), act'(g), bounds of both for an exact g, a bound on |act'| everywhere)."""
    a = g.abs()
    if name == "relu":
        return g.clamp(min=0), (g > 0).double(), torch.zeros_like(g), torch.zeros_like(g), 1.0
    if name == "gelu":
        phi, density = 0.5 * torch.erfc(-g / math.sqrt(2.0)), torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
        return (g * phi, phi + g * density, a * (PHI + UNDER) + 2 * U * (g * phi).abs(),
                PHI + (a * density) * (1.5 * g * g + 8) * U + 2 * U + (1 + a) * UNDER, 1.13)
    s, t = torch.sigmoid(g), torch.sigmoid(-g)
    rel = (1.5 * a + 10) * U
    if name == "sigmoid":
        return s, s * t, rel * s + UNDER, (2 * rel + U) * s * t + 2 * UNDER, 0.25
    return g * s, s + g * s * t, (rel + U) * a * s + a * UNDER, (rel + U) * s + (2 * rel + 3 * U) * a * s * t + (1 + 2 * a) * UNDER, 1.1


def glu(x, wg, wu, bg, bu, name):
    """(y, gate, up, bounds of the three)."""
    dtype, K = x.dtype, x.shape[1]
    x, wg, wu = x.double(), wg.double(), wu.double()
    zero = torch.zeros((), dtype=torch.float64, device=x.device)
    bg, bu = zero if bg is None else bg.double(), zero if bu is None else bu.double()
    g, u = x @ wg + bg, x @ wu + bu
    eg, eu = ((K + 4) * U * (x.abs() @ w.abs() + b.abs()) for w, b in ((wg, bg), (wu, bu)))
    a, _, ea, _, steep = act(name, g)
    ea = ea * 1.01 + 2 * U * eg + steep * eg
    y = a * u
    ey = ea * (u.abs() + eu) + a.abs() * eu + 2 * U * y.abs()
    slack = UB * 1.01 if dtype == torch.bfloat16 else U
    return y, g, u, ey + slack * (y.abs() + ey) + 1e-37, eg + slack * (g.abs() + eg), eu + slack * (u.abs() + eu)


def glu_grad(dy, x, wg, wu, gate, up, name):
    """(dx, dw_gate, dw_up, db_gate, db_up, bounds of the five), from the pre-activations as given."""
    dtype, (n, N) = x.dtype, dy.shape
    ub = UB if dtype == torch.bfloat16 else 0.0
    dy, x, wg, wu, g, u = (t.double() for t in (dy, x, wg, wu, gate, up))
    a, slope, ea, es, _ = act(name, g)
    dg, du = dy * u * slope, dy * a
    edg, edu = (dy * u).abs() * es + 3 * U * dg.abs(), dy.abs() * ea + 2 * U * du.abs()
    og, ou = edg * (1 + ub) + ub * dg.abs(), edu * (1 + ub) + ub * du.abs()        # as operands
    out = [dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du, dg.sum(0), du.sum(0)]
    err = [og @ wg.T.abs() + ou @ wu.T.abs() + (2 * N + 8) * U * (dg.abs() @ wg.T.abs() + du.abs() @ wu.T.abs())]
    err += [x.T.abs() @ e + (n + 16) * U * (x.T.abs() @ d.abs()) for e, d in ((og, dg), (ou, du))]
    err = [(e + out_round(t, dtype) * 1.01) * (1 + ub) + 1e-37 for e, t in zip(err, out)]
    err += [e.sum(0) + (n + 16) * U * d.abs().sum(0) + 1e-37 for e, d in ((edg, dg), (edu, du))]
    return (*out, *err)
