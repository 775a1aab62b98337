"""The parts of a block on histories that are timed: GMeta.seq_norm, causal GMeta.seq_attend, GMeta.seq_glu and their gradients.

A block of a history tower is norm -> attention of every event to the events up to it -> residual and norm -> gated feed-forward.
A batch holds many users' histories packed one behind the other.  A case is a dict of plain values.  `call` names the entry point:
  norm         GMeta.seq_norm: layer norm of the rows, of x + residual where there is one
  norm_grad    GMeta.seq_norm_grad: the gradients of rows, weight and bias, with what comes round the norm by the residual
  self         GMeta.seq_attend(causal=True): every event of a history attends to itself and the ones before it
  chunk        the same for the newest events of every user over a slot of the cache, which holds them already
  self_grad    GMeta.seq_attend_grad(causal=True)
  glu          GMeta.seq_glu: act(x Wg + bg) * (x Wu + bu)
  glu_grad     GMeta.seq_glu_grad: the gradients of rows, weights and biases, from the kept pre-activations
Widths and numbers of users are those of synth/configs.py and of the timed calls beside this file.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
EPS = 1e-5
OUT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _case(name, call, dtype, **kw):
    return dict(name=name, call=call, dtype=dtype, **kw)


def listed():
    return [
        # Serving: one event of each of 64 users, no residual yet: latency.
        _case("norm_few_fp32", "norm", "fp32", rows=64, channels=256, residual=0),
        # A training batch's events between attention and feed-forward: the residual is added on the way.
        _case("norm_rows_bf16", "norm", "bf16", rows=262_144, channels=512, residual=1),
        # Its gradient, with the residual's.
        _case("norm_grad_rows_bf16", "norm_grad", "bf16", rows=131_072, channels=512, residual=1),
        # Nothing round: a width that no vector load divides, few rows.
        _case("norm_grad_odd_fp32", "norm_grad", "fp32", rows=5_003, channels=845, residual=0),
        # Serving: the 16 newest events of 64 users over their slots, four query heads a key head.
        _case("chunk_users_bf16", "chunk", "bf16", users=64, queries=16, keys=4096, heads=8, kv_heads=2, dim=64, mask=0),
        # Encoding whole histories: the largest products.
        _case("self_long_bf16", "self", "bf16", users=32, keys=2048, heads=8, kv_heads=2, dim=128, mask=0),
        # Training: a batch's histories, some events taken out.
        _case("self_grad_users_bf16", "self_grad", "bf16", users=64, keys=1024, heads=8, kv_heads=4, dim=64, mask=1),
        # The same in fp32, short and ragged, a head of no round width.
        _case("self_grad_ragged_fp32", "self_grad", "fp32", users=37, keys=243, heads=4, kv_heads=4, dim=40, mask=1),
        # Serving: one event of each of 64 users: latency, the weights are what is read.
        _case("glu_few_bf16", "glu", "bf16", rows=64, d_in=512, d_out=1024, act="silu", bias=0, keep=0),
        # The forward pass of a training batch, pre-activations kept.
        _case("glu_rows_bf16", "glu", "bf16", rows=65_536, d_in=512, d_out=1024, act="silu", bias=0, keep=1),
        # Its gradient.
        _case("glu_grad_rows_bf16", "glu_grad", "bf16", rows=65_536, d_in=512, d_out=1024, act="silu", bias=0),
        # A small tower in fp32, nothing round, with biases.
        _case("glu_grad_odd_fp32", "glu_grad", "fp32", rows=3_001, d_in=132, d_out=260, act="gelu", bias=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    call = rng.choice(["norm", "norm_grad", "self", "chunk", "self_grad", "self_grad", "glu", "glu_grad"])
    dtype = rng.choice(["fp32", "bf16", "bf16"])
    if call in ("norm", "norm_grad"):
        return dict(call=call, dtype=dtype, rows=_log(rng, 1, 262_144), channels=rng.choice([_log(rng, 16, 2048), 64, 128, 256, 512, 1024]), residual=rng.choice([0, 1]))
    if call in ("glu", "glu_grad"):
        width = lambda: rng.choice([8 * _log(rng, 4, 128), 64, 128, 256, 512, 1024])  # noqa: E731
        c = dict(call=call, dtype=dtype, rows=_log(rng, 1, 65_536), d_in=width(), d_out=width(), act=rng.choice(["silu", "gelu", "sigmoid", "relu"]), bias=rng.choice([0, 1]))
        if call == "glu":
            c["keep"] = rng.choice([0, 1])
        return c
    kv = rng.choice([1, 2, 4])
    c = dict(call=call, dtype=dtype, users=_log(rng, 1, 256), keys=_log(rng, 16, 4096), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv, dim=rng.choice([32, 40, 64, 128]),
             mask=rng.choice([0, 1]))
    if call == "chunk":
        c["queries"] = _log(rng, 1, min(256, c["keys"]))
    return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (5e14 if case["dtype"] == "bf16" else 8e13)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        padded = c["users"] * c["heads"] * c.get("queries", c["keys"]) * c["keys"] if "users" in c else 0
        if _cost(c) <= most and padded <= 1.1e9:
            return c


# ---------------------------------------------------------------------------------------------- inputs
def _lengths(rng, n, longest):
    """Ragged: a new user has no history at all, one has the longest, the others lie evenly between; the seed says whose is whose."""
    s = np.rint(np.linspace(longest, max(1, longest // 8), n)).astype(np.int64)
    if n > 2:
        s[n // 2] = 0
    return rng.permutation(s)


def _offsets(lengths):
    return torch.from_numpy(np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)).cuda()


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * (seed % 1_000_000) + 29)
    rng = np.random.default_rng([seed % (1 << 32), 29])
    st, dt, call = SimpleNamespace(case=case), OUT[case["dtype"]], case["call"]
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    if call in ("norm", "norm_grad"):
        n, C = case["rows"], case["channels"]
        # (a residual stream: rows of unlike size, channels that stand out)
        stream = normal(n, C).mul_(torch.exp(normal(n, 1).mul_(0.5))).add_(normal(C).mul_(0.5)).to(dt)
        st.weight, st.bias = normal(C).mul_(0.1).add_(1.0), normal(C).mul_(0.1)
        st.residual = None
        if call == "norm":
            st.x = stream
            if case["residual"]:
                st.x, st.residual = normal(n, C).mul_(0.3).to(dt), stream
        else:
            st.x, st.dy = stream, normal(n, C).mul_(0.01).to(dt)
            f = stream.float()
            mean = f.mean(1)
            st.stats = torch.stack([mean, ((f - mean[:, None]).square().mean(1) + EPS).rsqrt()], 1)
            st.dsum = normal(n, C).mul_(0.01).to(dt) if case["residual"] else None
        return st
    if call in ("glu", "glu_grad"):
        n, K, N = case["rows"], case["d_in"], case["d_out"]
        st.x = normal(n, K).to(dt)                                            # (rows behind a norm)
        st.wg, st.wu = normal(K, N).mul_(K ** -0.5).to(dt), normal(K, N).mul_(K ** -0.5).to(dt)
        st.bg, st.bu = (normal(N).mul_(0.1), normal(N).mul_(0.1)) if case["bias"] else (None, None)
        if call == "glu_grad":
            st.gate, st.up = (t.to(dt) for t in _pre(st))
            st.dy = normal(n, N).mul_(0.01).to(dt)
        return st
    S, H, G, D = case["users"], case["heads"], case["kv_heads"], case["dim"]
    lk = _lengths(rng, S, case["keys"])
    st.longest_k, st.scale, st.k_lengths = case["keys"], 1.0 / math.sqrt(D), None
    if call == "chunk":     # every user has a slot of the cache, filled up to its length, the newest events' rows among them
        lk = np.maximum(lk, case["queries"])
        st.q_offsets, st.longest_q = _offsets(np.full(S, case["queries"])), case["queries"]
        st.k_offsets, st.k_lengths = _offsets(np.full(S, case["keys"])), torch.from_numpy(lk).cuda()
        Nq, Nk = S * case["queries"], S * case["keys"]
    else:
        st.q_offsets = st.k_offsets = _offsets(lk)
        st.longest_q, Nq, Nk = case["keys"], int(lk.sum()), int(lk.sum())
    st.q, st.k, st.v = normal(Nq, H, D).to(dt), normal(Nk, G, D).to(dt), normal(Nk, G, D).to(dt)
    st.key_mask = (torch.rand(Nk, device="cuda", generator=gen) < 0.9).to(torch.uint8) if case["mask"] else None
    if call == "self_grad":
        o, st.lse = _attend(st)
        st.o, st.dout = o.to(dt), normal(Nq, H, D).mul_(0.1).to(dt)
    return st


# ---------------------------------------------------------------------------------------------- the plain forms
def _norm(st):
    s = st.x.float() if st.residual is None else st.x.float() + st.residual.float()
    mean = s.mean(1, keepdim=True)
    rstd = torch.rsqrt(torch.square(s - mean).mean(1, keepdim=True) + EPS)
    return (s - mean) * rstd * st.weight + st.bias, s, torch.cat([mean, rstd], 1)


def _norm_grad(st):
    mean, rstd = st.stats[:, :1], st.stats[:, 1:]
    xh, dy = (st.x.float() - mean) * rstd, st.dy.float()
    g = dy * st.weight
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return dx if st.dsum is None else dx + st.dsum.float(), (dy * xh).sum(0), dy.sum(0)


def _pre(st):
    x = st.x.float()
    g, u = torch.matmul(x, st.wg.float()), torch.matmul(x, st.wu.float())
    return (g, u) if st.bg is None else (g + st.bg, u + st.bu)


def _phi(g):
    """The normal distribution's function, by the error function."""
    return 0.5 * (1.0 + torch.erf(g * math.sqrt(0.5)))


def _act(name, g):
    if name == "silu":
        return g * torch.sigmoid(g)
    if name == "gelu":
        return g * _phi(g)
    return torch.sigmoid(g) if name == "sigmoid" else torch.clamp(g, min=0.0)


def _act_slope(name, g):
    if name == "gelu":
        return _phi(g) + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)
    if name == "relu":
        return (g > 0).float()
    s = torch.sigmoid(g)
    return s + g * s * torch.sigmoid(-g) if name == "silu" else s * torch.sigmoid(-g)


def _glu_grad(st):
    act, g, u, dy, x = st.case["act"], st.gate.float(), st.up.float(), st.dy.float(), st.x.float()
    dg, du = dy * u * _act_slope(act, g), dy * _act(act, g)
    dx = torch.matmul(dg, st.wg.float().t().contiguous()) + torch.matmul(du, st.wu.float().t().contiguous())
    xt = x.t().contiguous()
    return dx, torch.matmul(xt, dg), torch.matmul(xt, du), dg.sum(0), du.sum(0)


def _place(offsets, n):
    """(sequence, position inside it) of n packed rows."""
    row = torch.arange(n, device="cuda")
    seq = torch.searchsorted(offsets, row, right=True) - 1
    return seq, row - offsets[seq]


def _pad(x, offsets, lengths, longest):
    """[sequences, longest, ...] in fp32, zeros behind every sequence's end."""
    at = torch.arange(longest, device="cuda")
    rows = (offsets[:-1, None] + at).clamp(max=max(len(x) - 1, 0))
    inside = at < lengths[:, None]
    return torch.where(inside.reshape(*inside.shape, *[1] * (x.dim() - 1)), x[rows].float(), 0.0)


def _scores(st):
    """Padded q, k, v [users, kv_heads, ., dim] (a key head's query heads side by side) and the scores, -infinity where a key does not count or lies
    behind the query's own place, which is counted from the end of both."""
    c = st.case
    S, H, G, D = c["users"], c["heads"], c["kv_heads"], c["dim"]
    lq = st.q_offsets[1:] - st.q_offsets[:-1]
    lk = st.k_offsets[1:] - st.k_offsets[:-1] if st.k_lengths is None else st.k_lengths
    keep = torch.ones(len(st.k), dtype=torch.bool, device="cuda") if st.key_mask is None else st.key_mask != 0
    at_k = torch.arange(st.longest_k, device="cuda")
    kept = (at_k < lk[:, None]) & (_pad(keep[:, None], st.k_offsets, lk, st.longest_k)[..., 0] > 0)
    seen = at_k <= (torch.arange(st.longest_q, device="cuda") + (lk - lq)[:, None])[..., None]                     # [users, queries, keys]
    counts = (kept[:, None] & seen).repeat_interleave(H // G, 1)[:, None]
    rows = lambda t: _pad(t, st.q_offsets, lq, st.longest_q).reshape(S, -1, G, H // G, D).permute(0, 2, 1, 3, 4).reshape(S, G, -1, D)  # noqa: E731
    keys = lambda t: torch.where(kept[:, None, :, None], _pad(t, st.k_offsets, lk, st.longest_k).permute(0, 2, 1, 3), 0.0)  # noqa: E731
    q, k, v = rows(st.q), keys(st.k), keys(st.v)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st.scale
    return q, k, v, torch.where(counts, s, -math.inf), rows


def _packed(st, t):
    """[users, kv_heads, rows, ...] -> [all queries, heads, ...]"""
    c = st.case
    t = t.reshape(c["users"], c["kv_heads"], st.longest_q, c["heads"] // c["kv_heads"], *t.shape[3:])
    seq, pos = _place(st.q_offsets, len(st.q))
    return t.transpose(1, 2)[seq, pos].reshape(len(st.q), c["heads"], *t.shape[4:])


def _attend(st):
    _, _, v, s, _ = _scores(st)
    top = s.amax(3, keepdim=True)
    p = torch.exp(s - torch.where(top > -math.inf, top, 0.0))
    total = p.sum(3, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total > 0, total, 1.0)
    return _packed(st, o), _packed(st, (torch.log(total) + top)[..., 0])


def _attend_grad(st):
    q, k, v, s, rows = _scores(st)
    lse = rows(st.lse[..., None].expand(*st.lse.shape, st.case["dim"]))[..., :1]
    p = torch.exp(s - torch.where(lse > -math.inf, lse, 0.0))
    do, o = rows(st.dout), rows(st.o)
    ds = p * (torch.matmul(do, v.transpose(2, 3).contiguous()) - (do * o).sum(3, keepdim=True)) * st.scale
    dq, dk, dv = torch.matmul(ds, k), torch.matmul(ds.transpose(2, 3).contiguous(), q), torch.matmul(p.transpose(2, 3).contiguous(), do)
    seq, pos = _place(st.k_offsets, len(st.k))
    return _packed(st, dq), dk.transpose(1, 2)[seq, pos], dv.transpose(1, 2)[seq, pos]


def _run_plain(st):
    call, dt = st.case["call"], OUT[st.case["dtype"]]
    if call == "norm":
        y, s, stats = _norm(st)
        return [y.to(dt), s.to(dt), stats]
    if call == "norm_grad":
        dx, dw, db = _norm_grad(st)
        return [dx.to(dt), dw, db]
    if call == "glu":
        g, u = _pre(st)
        y = (_act(st.case["act"], g) * u).to(dt)
        return [y, g.to(dt), u.to(dt)] if st.case["keep"] else [y]
    if call == "glu_grad":
        dx, dwg, dwu, dbg, dbu = _glu_grad(st)
        return [dx.to(dt), dwg.to(dt), dwu.to(dt)] + ([dbg, dbu] if st.case["bias"] else [])
    if call == "self_grad":
        return [t.to(dt) for t in _attend_grad(st)]
    o, lse = _attend(st)
    return [o.to(dt), lse]


# ---------------------------------------------------------------------------------------------- the framework's calls
_context = None


def _gm():
    """The handle a program keeps: a context whose calls return once enqueued, as work between other work of a stream."""
    global _context
    if _context is None:
        from paper_2401_04338_amd import GMeta
        _context = GMeta(1, [1000], 64, 13, [77, 64, 1], workspace_bytes=1 << 30)
        _context.configure("wait", 0)
    return _context


def run(st):
    if not own:
        return _run_plain(st)
    gm, c = _gm(), st.case
    if c["call"] == "norm":
        return list(gm.seq_norm(st.x, st.weight, st.bias, eps=EPS, residual=st.residual))
    if c["call"] == "norm_grad":
        return list(gm.seq_norm_grad(st.dy, st.x, st.stats, st.weight, dsum=st.dsum))
    if c["call"] == "glu":
        out = gm.seq_glu(st.x, st.wg, st.wu, c["act"], b_gate=st.bg, b_up=st.bu, keep=bool(c["keep"]))
        return list(out) if c["keep"] else [out]
    if c["call"] == "glu_grad":
        out = gm.seq_glu_grad(st.dy, st.x, st.wg, st.wu, st.gate, st.up, c["act"], bias=bool(c["bias"]))
        return list(out) if c["bias"] else list(out[:3])
    kw = dict(scale=st.scale, key_mask=st.key_mask, causal=True)
    if c["call"] == "self_grad":
        return list(gm.seq_attend_grad(st.dout, st.q, st.k, st.v, st.o, st.lse, st.q_offsets, st.k_offsets, st.longest_q, st.longest_k, **kw))
    return list(gm.seq_attend(st.q, st.k, st.v, st.q_offsets, st.k_offsets, st.longest_q, st.longest_k, k_lengths=st.k_lengths, **kw))


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _exact_attend(st, grad):
    """User by user and head by head."""
    c = st.case
    qo, ko = st.q_offsets.tolist(), st.k_offsets.tolist()
    lk = [b - a for a, b in zip(ko[:-1], ko[1:])] if st.k_lengths is None else st.k_lengths.tolist()
    o = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), torch.zeros(st.k.shape, dtype=torch.float64, device="cuda"), torch.zeros(st.k.shape, dtype=torch.float64, device="cuda")
    for u in range(c["users"]):
        lq = qo[u + 1] - qo[u]
        n = torch.arange(lk[u], device="cuda")
        if st.key_mask is not None:
            n = n[st.key_mask[ko[u] + n] != 0]
        if not len(n) or not lq:
            continue
        hidden = n[None] > torch.arange(lk[u] - lq, lk[u], device="cuda")[:, None]
        some = ~hidden.all(1, keepdim=True)
        rows, n = slice(qo[u], qo[u + 1]), ko[u] + n
        for hd in range(c["heads"]):
            g = hd // (c["heads"] // c["kv_heads"])
            q, k, v = st.q[rows, hd].double(), st.k[n, g].double(), st.v[n, g].double()
            s = (q @ k.T * st.scale).masked_fill_(hidden, -math.inf)
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - torch.where(some, l[:, None], 0.0))
            o[rows, hd], lse[rows, hd] = p @ v, l
            if grad:
                do = st.dout[rows, hd].double()
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * st.scale
                dq[rows, hd] = ds @ k
                dk[n, g] += ds.T @ q
                dv[n, g] += p.T @ do
    return [dq, dk, dv] if grad else [o, lse]


def _exact_act(name, g):
    """(value, slope)"""
    if name == "relu":
        return g * (g > 0), (g > 0).double()
    if name == "gelu":
        phi = 0.5 * torch.erfc(-g / math.sqrt(2.0))
        return g * phi, phi + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    s, t = 1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))
    return (g * s, s * (1 + g * t)) if name == "silu" else (s, s * t)


def _exact_glu(st, grad):
    x, wg, wu, act = st.x.double(), st.wg.double(), st.wu.double(), st.case["act"]
    if not grad:
        g, u = x @ wg, x @ wu
        if st.bg is not None:
            g, u = g + st.bg.double(), u + st.bu.double()
        y = _exact_act(act, g)[0] * u
        return [y, g, u] if st.case["keep"] else [y]
    a, slope = _exact_act(act, st.gate.double())
    d = st.dy.double()
    dg, du = d * st.up.double() * slope, d * a
    out = [dg @ wg.T + du @ wu.T, x.T @ dg, x.T @ du]
    return out + [dg.sum(0), du.sum(0)] if st.case["bias"] else out


def _exact_norm(st):
    s = st.x.double()
    if st.residual is not None:
        s = s + st.residual.double()
    var, mean = torch.var_mean(s, dim=1, correction=0, keepdim=True)
    xh = (s - mean) / torch.sqrt(var + EPS)
    return [xh * st.weight.double() + st.bias.double(), s, torch.cat([mean, 1 / torch.sqrt(var + EPS)], 1)]


def _exact_norm_grad(st):
    mean, rstd = st.stats.double().split(1, 1)
    n, xh, d = st.case["channels"], (st.x.double() - mean) * rstd, st.dy.double()
    g = d * st.weight.double()
    dx = (n * g - g.sum(1, keepdim=True) - xh * (g * xh).sum(1, keepdim=True)) * (rstd / n)
    return [dx if st.dsum is None else dx + st.dsum.double(), (d * xh).sum(0), d.sum(0)]


def exact(case, seed):
    call, st = case["call"], prepare(case, seed)
    if call == "norm":
        return _exact_norm(st)
    if call == "norm_grad":
        return _exact_norm_grad(st)
    if call in ("glu", "glu_grad"):
        return _exact_glu(st, call == "glu_grad")
    return _exact_attend(st, call == "self_grad")


# ---------------------------------------------------------------------------------------------- what a pass has to do
def work(case):
    """Operands once, outputs once; the products that no form can leave out (attention: two forward, five backward, over the keys that a query sees), a
    few operations an element elsewhere."""
    s = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["call"] in ("norm", "norm_grad"):
        n, C, r = case["rows"], case["channels"], case["residual"]
        if case["call"] == "norm":
            return {"bytes": n * C * s * (2 + 2 * r) + n * 8 + C * 8, "flops": 8.0 * n * C}
        return {"bytes": n * C * s * (3 + r) + n * 8 + C * 12, "flops": 14.0 * n * C}
    if case["call"] in ("glu", "glu_grad"):
        n, K, N = case["rows"], case["d_in"], case["d_out"]
        if case["call"] == "glu":
            return {"bytes": s * (n * K + 2 * K * N + n * N * (1 + 2 * case["keep"])) + 8 * N * case["bias"], "flops": 4.0 * n * K * N}
        return {"bytes": s * (2 * n * K + 4 * K * N + 3 * n * N) + 8 * N * case["bias"], "flops": 8.0 * n * K * N}
    u, H, G, D = case["users"], case["heads"], case["kv_heads"], case["dim"]
    lens = np.linspace(case["keys"], max(1, case["keys"] // 8), u)
    if case["call"] == "chunk":
        lens, lq = np.maximum(lens, case["queries"]), np.full(u, float(case["queries"]))
    else:
        lq = lens
    pairs = float((lq * (lens - (lq - 1) / 2)).sum()) * H * (0.9 if case["mask"] else 1.0)
    nq, nk, rows = float(lq.sum()) * H * D * s, float(lens.sum()) * G * D * s, float(lq.sum()) * H * 4
    if case["call"] == "self_grad":
        return {"bytes": 4 * nq + 4 * nk + rows, "flops": 10.0 * pairs * D}
    return {"bytes": 2 * nq + 2 * nk + rows, "flops": 4.0 * pairs * D}
