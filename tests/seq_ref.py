"""The calls on histories in 64 bits, on the CPU, each with a bound on the error of fp32 arithmetic (and of bf16 operands and
outputs where the tensors are bf16), element by element, from the standard model of rounding: a computed sum of n products is off
by at most (n + 1) u times the sum of their magnitudes."""
from __future__ import annotations

import torch

U = 2.0 ** -24        # unit roundoff of fp32
UB = 2.0 ** -8        # of bf16: 8 significant bits, as 24 of fp32


def out_round(y, dtype):
    return UB * y.abs() * 1.01 if dtype == torch.bfloat16 else U * y.abs()


def embed_grad(grad, tokens, n_rows, scale):
    """(rows, sums, bound): sums of m terms, then one product."""
    g, tok = grad.double(), tokens.long()
    rows = torch.unique(tok[tok >= 0])
    sums, mags, counts = (torch.zeros(n_rows, g.shape[1], dtype=torch.float64) for _ in range(3))
    keep = tok >= 0
    sums.index_add_(0, tok[keep], g[keep])
    mags.index_add_(0, tok[keep], g[keep].abs())
    counts.index_add_(0, tok[keep], torch.ones_like(g[keep]))
    return rows, scale * sums[rows], ((counts + 2) * U * abs(scale) * mags)[rows]


# A gate's relative error: |g| log2(e) is rounded (|g| <= 12 here: 12 u in the exponential), the exponential and the reciprocal
# are good to one ulp (2 u each), a sum and a product: 18 u.  A step adds a rounding or two, and steps are combined in pieces, whose
# coefficients carry their own: at most as much again.
STEP = 40 * U


def scan(x, gate, lengths, h0):
    """(h, last, bounds of both) by the recurrence, a step at a time; the bound runs along."""
    x, a, b = x.double(), torch.sigmoid(gate.double()), torch.sigmoid(-gate.double())
    h, bound = torch.zeros_like(x), torch.zeros_like(x)
    S, C = len(lengths), x.shape[1]
    last, last_bound = torch.zeros(S, C, dtype=torch.float64), torch.zeros(S, C, dtype=torch.float64)
    at = 0
    for s, n in enumerate(lengths):
        y = torch.zeros(C, dtype=torch.float64) if h0 is None else h0[s].double()
        e = torch.zeros(C, dtype=torch.float64)
        for t in range(at, at + n):
            e = a[t] * e + STEP * (a[t] * y.abs() + b[t] * x[t].abs())
            y = a[t] * y + b[t] * x[t]
            h[t], bound[t] = y, e
        last[s], last_bound[s] = y, e
        at += n
    return h, last, bound, last_bound


def scan_grad(dh, x, gate, h, lengths, h0, dlast):
    """(dx, dgate, dh0) and their bounds, from h as given."""
    x, h, dh, a, b = x.double(), h.double(), dh.double(), torch.sigmoid(gate.double()), torch.sigmoid(-gate.double())
    dx, dg, ex, eg = (torch.zeros_like(x) for _ in range(4))
    S, C = len(lengths), x.shape[1]
    d0, e0 = torch.zeros(S, C, dtype=torch.float64), torch.zeros(S, C, dtype=torch.float64)
    at = 0
    for s, n in enumerate(lengths):
        c = torch.zeros(C, dtype=torch.float64) if dlast is None else dlast[s].double()
        e = torch.zeros(C, dtype=torch.float64)
        first = torch.zeros(C, dtype=torch.float64) if h0 is None else h0[s].double()
        for t in reversed(range(at, at + n)):
            before = h[t - 1] if t > at else first
            d = dh[t] + c
            k = a[t] * b[t]
            dx[t], dg[t] = b[t] * d, d * (before - x[t]) * k
            ed = e + U * (dh[t].abs() + c.abs())
            ex[t] = b[t] * ed + STEP * dx[t].abs()
            eg[t] = k * (ed * (before - x[t]).abs() + U * d.abs() * (before.abs() + x[t].abs())) + 2 * STEP * dg[t].abs()
            e = a[t] * ed + STEP * a[t] * (dh[t].abs() + c.abs())
            c = a[t] * d
        d0[s], e0[s] = c, e
        at += n
    return dx, dg, d0, ex, eg, e0


def _pairs(q, k, q_off, k_start, k_len, mask):
    """Per sequence and head: the rows, the keys that count."""
    H, G = q.shape[1], k.shape[1]
    for s in range(len(q_off) - 1):
        keys = torch.arange(k_start[s], k_start[s] + k_len[s])
        if mask is not None:
            keys = keys[mask[keys] != 0]
        for h in range(H):
            yield slice(q_off[s], q_off[s + 1]), keys, h, h // (H // G)


def _score(q, k, scale):
    """Scores and the error of their exponential: the product's, the rounding of scale * log2(e) and of its product with the score,
    and the exponential's own."""
    s = q @ k.T * scale
    return s, U * ((q.shape[1] + 4) * scale * (q.abs() @ k.abs().T) + 4 * s.abs() + 8)


def attend(q, k, v, q_off, k_start, k_len, scale, mask):
    dtype = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    o, eo = torch.zeros_like(q), torch.zeros_like(q)
    lse = torch.full(q.shape[:2], -float("inf"), dtype=torch.float64)
    el = torch.zeros(q.shape[:2], dtype=torch.float64)
    for rows, keys, h, g in _pairs(q, k, q_off, k_start, k_len, mask):
        if len(keys) == 0 or rows.start == rows.stop:
            continue
        s, es = _score(q[rows, h], k[keys, g], scale)
        lse[rows, h] = torch.logsumexp(s, 1)
        p = torch.exp(s - lse[rows, h][:, None])
        mean = (p * es).sum(1, keepdim=True)
        # (each rescaling to a new maximum costs an exponential and a product: at most one per 32 keys and one per piece)
        es = es + mean + (3 * len(keys) + 64) * U
        w = p * (es + (UB if dtype == torch.bfloat16 else 0.0))
        o[rows, h] = p @ v[keys, g]
        eo[rows, h] = w @ v[keys, g].abs() + out_round(o[rows, h], dtype)
        el[rows, h] = mean[:, 0] + (len(keys) + 64) * U + 4 * U * lse[rows, h].abs() + 4 * U * s.abs().amax(1)
    return o, lse, eo, el


def attend_grad(dout, q, k, v, o, lse, q_off, k_start, k_len, scale, mask):
    """From o and lse as given."""
    dtype = q.dtype
    ub = UB if dtype == torch.bfloat16 else 0.0
    dout, q, k, v, o, lse = (t.double() for t in (dout, q, k, v, o, lse))
    dq, dk, dv, eq, ek, ev = (torch.zeros_like(t) for t in (q, k, v, q, k, v))
    rk = torch.zeros_like(k)
    n_rows = torch.zeros(len(k), dtype=torch.float64)
    for rows, keys, h, g in _pairs(q, k, q_off, k_start, k_len, mask):
        n = len(keys)
        if n == 0 or rows.start == rows.stop:
            continue
        D, m = q.shape[2], rows.stop - rows.start
        qr, kr, vr, do, orow = q[rows, h], k[keys, g], v[keys, g], dout[rows, h], o[rows, h]
        s, es = _score(qr, kr, scale)
        p = torch.exp(s - lse[rows, h][:, None])
        es = es + 4 * U * lse[rows, h].abs()[:, None]
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


def within(got, want, bound, what=""):
    """|got - want| <= bound everywhere; infinities and NaN in the same places."""
    g, w = got.detach().cpu().double(), want.double()
    assert g.shape == w.shape, (what, g.shape, w.shape)
    fine = torch.isfinite(w)
    assert torch.equal(torch.isnan(g), torch.isnan(w)), f"{what}: NaN elsewhere"
    assert torch.equal(g[~fine & ~torch.isnan(w)], w[~fine & ~torch.isnan(w)]), f"{what}: infinities elsewhere"
    off = (g - w).abs()[fine] - bound[fine] - 1e-37
    assert not (off > 0).any(), f"{what}: {int((off > 0).sum())} of {off.numel()} values off, worst by {float(off.max()):.3g} over a bound of {float(bound[fine].max()):.3g}"
