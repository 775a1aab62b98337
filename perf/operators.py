"""The operators of a user's history that are timed: the calls of GMeta.seq_* over the range of sizes they are used at.

A history is an ordered list of item tokens of any length; a batch holds many users' histories, packed one behind the other
(offsets say where each begins).  A case is a dict of plain values.  `call` names the entry point:
  embed        GMeta.seq_embed: rows of a table, scaled, one per token
  embed_grad   GMeta.seq_embed_grad: their gradient as a coalesced row list (form "list"), or added to a table (form "table")
  scan         GMeta.seq_scan: the gated linear recurrence over every history
  scan_grad    GMeta.seq_scan_grad: its gradients
  scan_step    GMeta.seq_scan_step: one token of every user, states in place
  attend       GMeta.seq_attend: candidates' queries over the encoder's states
  attend_grad  GMeta.seq_attend_grad: the gradients of queries, keys and values
Table sizes, widths and numbers of users are those of synth/configs.py and of the timed calls beside this file.
"""
import math
from types import SimpleNamespace

import numpy as np
import torch

own = False
SCALE = 1.7   # of the lookups: a constant that is no power of two
OUT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def _case(name, call, dtype, **kw):
    return dict(name=name, call=call, dtype=dtype, **kw)


def listed():
    return [
        # A handful of new tokens to score: latency of a lookup.
        _case("embed_few_fp32", "embed", "fp32", tokens=2048, rows=100_000, dim=32, zipf=1.05),
        # The histories of a training batch, 256 thousand events twice over: inputs and gates in one row of 128.
        _case("embed_histories_bf16", "embed", "bf16", tokens=1_000_000, rows=1_000_000, dim=128, zipf=1.05),
        # The gradient of those rows, listed.
        _case("embed_grad_histories_bf16", "embed_grad", "bf16", tokens=1_000_000, rows=1_000_000, dim=128, zipf=1.1, form="list"),
        # Nothing round: a small table, updated in place.
        _case("embed_update_odd_fp32", "embed_grad", "fp32", tokens=61_003, rows=7_001, dim=36, zipf=1.05, form="table"),
        # Serving: one event of each of 512 users.
        _case("scan_step_users_bf16", "scan_step", "bf16", users=512, channels=256),
        # Training: 1,024 users' histories of 64 to 512 events.
        _case("scan_users_bf16", "scan", "bf16", users=1024, longest=512, channels=256, state=1),
        # Few long logs: the parallelism has to come from the time axis.
        _case("scan_grad_long_bf16", "scan_grad", "bf16", users=4, longest=40_000, channels=256, state=0),
        # Ragged histories, odd number of channels, carried states.
        _case("scan_grad_ragged_fp32", "scan_grad", "fp32", users=201, longest=243, channels=100, state=1),
        # Serving: one candidate a user over a cache of long histories, four query heads a key head.
        _case("attend_one_bf16", "attend", "bf16", users=64, queries=1, keys=4096, heads=8, kv_heads=2, dim=64, mask=0, cache=1),
        # Ranking long candidate lists over long histories: the largest products.
        _case("attend_long_bf16", "attend", "bf16", users=64, queries=512, keys=2048, heads=8, kv_heads=2, dim=128, mask=0, cache=0),
        # Training: candidates of a batch over their users' histories, some events taken out.
        _case("attend_grad_users_bf16", "attend_grad", "bf16", users=64, queries=256, keys=1024, heads=8, kv_heads=4, dim=64, mask=1, cache=0),
        # The same in fp32, short and ragged, a head of no round width.
        _case("attend_grad_ragged_fp32", "attend_grad", "fp32", users=37, queries=61, keys=243, heads=4, kv_heads=4, dim=40, mask=1, cache=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _draw_once(rng):
    call, dtype = rng.choice(["embed", "embed_grad", "embed_grad", "scan", "scan_grad", "scan_step", "attend", "attend", "attend_grad", "attend_grad"]), rng.choice(["fp32", "bf16"])
    if call in ("embed", "embed_grad"):
        c = _case("", call, dtype, tokens=_log(rng, 1_000, 1_000_000), rows=_log(rng, 1_000, 1_000_000), dim=rng.choice([16, 32, 36, 64, 100, 128]),
                  zipf=rng.choice([0.0, 1.05, 1.1]))
        if call == "embed_grad":
            c["form"] = rng.choice(["list", "table"])
    elif call == "scan_step":
        c = _case("", call, dtype, users=_log(rng, 1, 4096), channels=rng.choice([32, 64, 100, 256]))
    elif call in ("scan", "scan_grad"):
        c = _case("", call, dtype, users=_log(rng, 1, 1024), longest=_log(rng, 16, 40_000), channels=rng.choice([32, 64, 100, 256]), state=rng.choice([0, 1]))
    else:
        kv = rng.choice([1, 2, 4])
        c = _case("", call, dtype, users=_log(rng, 1, 256), queries=_log(rng, 1, 512), keys=_log(rng, 16, 4096), heads=kv * rng.choice([1, 2, 4]), kv_heads=kv,
                  dim=rng.choice([32, 40, 64, 128]), mask=rng.choice([0, 1]), cache=rng.choice([0, 1]) if call == "attend" else 0)
    del c["name"]
    return c


def _cost(case):
    w = work(case)
    return w["bytes"] / 4e12 + w["flops"] / (5e14 if case["dtype"] == "bf16" else 8e13)


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_once(rng)
        padded = c["users"] * c["heads"] * c["queries"] * c["keys"] if c["call"].startswith("attend") else c.get("users", 0) * c.get("longest", 0) * c.get("channels", 0)
        if _cost(c) <= most and padded <= 5.5e8:
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


def _tokens(case, gen):
    """Item tokens by bounded Zipf, the hot ranks spread over the table; one in 64 is padding (-1)."""
    n, R = case["tokens"], case["rows"]
    p = torch.arange(1, R + 1, dtype=torch.float64, device="cuda") ** -case["zipf"]
    cdf = torch.cumsum(p, 0)
    rank = torch.searchsorted(cdf / cdf[-1], torch.rand(n, dtype=torch.float64, device="cuda", generator=gen)).clamp_(max=R - 1)
    mult = 2_654_435_761 % R | 1
    while math.gcd(mult, R) != 1:
        mult += 2
    row = rank * mult % R
    return torch.where(torch.rand(n, device="cuda", generator=gen) < 1 / 64, -1, row).to(torch.int32)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(1_000_003 * (seed % 1_000_000) + 17)
    rng = np.random.default_rng([seed % (1 << 32), 17])
    st, dt = SimpleNamespace(case=case), OUT[case["dtype"]]
    normal = lambda *s: torch.randn(*s, device="cuda", generator=gen)  # noqa: E731
    if case["call"] in ("embed", "embed_grad"):
        n, R, D = case["tokens"], case["rows"], case["dim"]
        st.tokens = _tokens(case, gen)
        if case["call"] == "embed":
            st.table = normal(R, D).mul_(0.05)
        else:
            st.grad = normal(n, D).mul_(0.01).to(dt)
            if case["form"] == "table":
                st.table = torch.zeros(R, D, device="cuda")
            else:
                cap = min(n, R)
                st.out = dict(emb_rows=torch.zeros(cap, dtype=torch.int64, device="cuda"), emb_grad=torch.zeros(cap, D, device="cuda"),
                              n_emb_rows=torch.zeros(1, dtype=torch.int64, device="cuda"), capacity=cap)
        return st
    if case["call"] == "scan_step":
        S, C = case["users"], case["channels"]
        st.x, st.gate, st.state = normal(S, C).to(dt), normal(S, C).add_(2.0).to(dt), normal(S, C).mul_(0.3)
        return st
    if case["call"] in ("scan", "scan_grad"):
        S, C = case["users"], case["channels"]
        lens = _lengths(rng, S, case["longest"])
        st.offsets, st.longest, N = _offsets(lens), case["longest"], int(lens.sum())
        st.x, st.gate = normal(N, C).to(dt), normal(N, C).mul_(1.5).add_(2.0).to(dt)   # (a memory of some ten events, up to hundreds)
        st.h0 = normal(S, C).mul_(0.3) if case["state"] else None
        if case["call"] == "scan_grad":
            st.h = _scan(st.x, st.gate, st.offsets, st.longest, st.h0)[0].to(dt)
            st.dh, st.dlast = normal(N, C).mul_(0.01).to(dt), normal(S, C).mul_(0.01) if case["state"] else None
        return st
    S, H, G, D = case["users"], case["heads"], case["kv_heads"], case["dim"]
    lq, lk = _lengths(rng, S, case["queries"]), _lengths(rng, S, case["keys"])
    if case["queries"] == 1 or case["cache"]:
        lq[:] = case["queries"]
    st.q_offsets, st.longest_q, st.longest_k, st.scale = _offsets(lq), case["queries"], case["keys"], 1.0 / math.sqrt(D)
    st.k_lengths = None
    if case["cache"]:     # every user has a slot of the cache, filled up to its length
        st.k_offsets, st.k_lengths = _offsets(np.full(S, case["keys"])), torch.from_numpy(lk.astype(np.int64)).cuda()
        Nk = S * case["keys"]
    else:
        st.k_offsets, Nk = _offsets(lk), int(lk.sum())
    st.q, st.k, st.v = normal(int(lq.sum()), H, D).to(dt), normal(Nk, G, D).to(dt), normal(Nk, G, D).to(dt)
    st.key_mask = (torch.rand(Nk, device="cuda", generator=gen) < 0.9).to(torch.uint8) if case["mask"] else None
    if case["call"] == "attend_grad":
        o, st.lse = _attend(st)
        st.o, st.dout = o.to(dt), normal(int(lq.sum()), H, D).mul_(0.1).to(dt)
    return st


# ---------------------------------------------------------------------------------------------- the plain forms
def _embed(table, tokens):
    return torch.where((tokens >= 0)[:, None], table[tokens.clamp(min=0)] * SCALE, 0.0)


def _embed_grad(st):
    keep = st.tokens >= 0
    tok, g = st.tokens[keep].long(), st.grad[keep].float() * SCALE
    if st.case["form"] == "table":
        return st.table.index_add_(0, tok, g)
    rows, place = torch.unique(tok, return_inverse=True)
    o = st.out
    o["emb_rows"][:len(rows)] = rows
    o["emb_grad"][:len(rows)] = torch.zeros(len(rows), g.shape[1], device="cuda").index_add_(0, place, g)
    o["n_emb_rows"].fill_(len(rows))
    return [o["emb_rows"], o["emb_grad"], o["n_emb_rows"]]


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


def _doubled(a, b):
    """y_t = a_t y_{t-1} + b_t along the second axis by doubling: after the step of d, (a, b) span 2 d places."""
    d, n = 1, a.shape[1]
    while d < n:
        b2, a2 = b.clone(), a.clone()
        b2[:, d:] += a[:, d:] * b[:, :n - d]
        a2[:, d:] *= a[:, :n - d]
        a, b, d = a2, b2, 2 * d
    return a, b


def _scan(x, gate, offsets, longest, h0):
    lens = offsets[1:] - offsets[:-1]
    seq, pos = _place(offsets, len(x))
    xp, gp = _pad(x, offsets, lens, longest), _pad(gate, offsets, lens, longest)
    A, B = _doubled(torch.sigmoid(gp), torch.sigmoid(-gp) * xp)
    h = B if h0 is None else A * h0[:, None] + B
    last = h[torch.arange(len(lens), device="cuda"), (lens - 1).clamp(min=0)]
    return h[seq, pos], torch.where((lens > 0)[:, None], last, 0.0 if h0 is None else h0)


def _scan_grad(st):
    offsets, longest = st.offsets, st.longest
    lens = offsets[1:] - offsets[:-1]
    seq, pos = _place(offsets, len(st.x))
    x, g, h, dh = (_pad(t, offsets, lens, longest) for t in (st.x, st.gate, st.h, st.dh))
    a, na = torch.sigmoid(g), torch.sigmoid(-g)
    inside = (torch.arange(longest, device="cuda") < lens[:, None])[..., None]
    a = torch.where(inside, a, 1.0)        # (what lies behind a sequence's end hands the carry on)
    zero = torch.zeros(len(lens), 1, x.shape[2], device="cuda")
    A, B = _doubled(a.flip(1), (a * dh).flip(1))
    c = B if st.dlast is None else A * st.dlast[:, None] + B
    c = c.flip(1)                          # c_t = a_t (dh_t + c_{t+1})
    d = dh + torch.cat([c[:, 1:], zero if st.dlast is None else st.dlast[:, None]], 1)
    before = torch.cat([zero if st.h0 is None else st.h0[:, None], h[:, :-1]], 1)
    dx, dg = na * d, d * (before - x) * a * na
    return dx[seq, pos], dg[seq, pos], c[:, 0] if st.h0 is not None else None


def _scores(st):
    """Padded q, k, v [users, kv_heads, ., dim] (a key head's query heads side by side), the scores and which keys count."""
    c = st.case
    S, H, G, D = c["users"], c["heads"], c["kv_heads"], c["dim"]
    lq = st.q_offsets[1:] - st.q_offsets[:-1]
    lk = st.k_offsets[1:] - st.k_offsets[:-1] if st.k_lengths is None else st.k_lengths
    keep = torch.ones(len(st.k), dtype=torch.bool, device="cuda") if st.key_mask is None else st.key_mask != 0
    kept = (torch.arange(st.longest_k, device="cuda") < lk[:, None]) & (_pad(keep[:, None], st.k_offsets, lk, st.longest_k)[..., 0] > 0)
    rows = lambda t: _pad(t, st.q_offsets, lq, st.longest_q).reshape(S, -1, G, H // G, D).permute(0, 2, 1, 3, 4).reshape(S, G, -1, D)  # noqa: E731
    keys = lambda t: torch.where(kept[:, None, :, None], _pad(t, st.k_offsets, lk, st.longest_k).permute(0, 2, 1, 3), 0.0)  # noqa: E731
    q, k, v = rows(st.q), keys(st.k), keys(st.v)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()) * st.scale
    return q, k, v, torch.where(kept[:, None, None], s, -math.inf), rows


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
    if call == "embed":
        return _embed(st.table, st.tokens).to(dt)
    if call == "embed_grad":
        return _embed_grad(st)
    if call == "scan_step":
        a, b = torch.sigmoid(st.gate.float()), torch.sigmoid(-st.gate.float())
        st.state.mul_(a).add_(b * st.x.float())
        return [st.state.to(dt), st.state]
    if call == "scan":
        h, last = _scan(st.x, st.gate, st.offsets, st.longest, st.h0)
        return [h.to(dt), last]
    if call == "scan_grad":
        dx, dg, dh0 = _scan_grad(st)
        return [dx.to(dt), dg.to(dt), dh0]
    if call == "attend":
        o, lse = _attend(st)
        return [o.to(dt), lse]
    return [t.to(dt) for t in _attend_grad(st)]


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
    gm, c, dt = _gm(), st.case, OUT[st.case["dtype"]]
    if c["call"] == "embed":
        return gm.seq_embed(st.table, st.tokens, SCALE, dtype=dt)
    if c["call"] == "embed_grad":
        if c["form"] == "table":
            gm.seq_embed_grad(st.grad, st.tokens, c["rows"], SCALE, table=st.table)
            return st.table
        o = gm.seq_embed_grad(st.grad, st.tokens, c["rows"], SCALE, out=st.out)
        return [o["emb_rows"], o["emb_grad"], o["n_emb_rows"]]
    if c["call"] == "scan_step":
        return [gm.seq_scan_step(st.x, st.gate, st.state), st.state]
    if c["call"] == "scan":
        return list(gm.seq_scan(st.x, st.gate, st.offsets, st.longest, h0=st.h0))
    if c["call"] == "scan_grad":
        return list(gm.seq_scan_grad(st.dh, st.x, st.gate, st.h, st.offsets, st.longest, h0=st.h0, dlast=st.dlast))
    kw = dict(scale=st.scale, key_mask=st.key_mask)
    if c["call"] == "attend":
        return list(gm.seq_attend(st.q, st.k, st.v, st.q_offsets, st.k_offsets, st.longest_q, st.longest_k, k_lengths=st.k_lengths, **kw))
    return list(gm.seq_attend_grad(st.dout, st.q, st.k, st.v, st.o, st.lse, st.q_offsets, st.k_offsets, st.longest_q, st.longest_k, **kw))


# ---------------------------------------------------------------------------------------------- the same in 64 bits
def _exact_scan(st, grad):
    """A step of all users at a time, users in the order they come."""
    off = st.offsets.tolist()
    lens = [b - a for a, b in zip(off[:-1], off[1:])]
    x, e = st.x.double(), torch.exp(-st.gate.double())
    a, b = 1 / (1 + e), e / (1 + e)
    S, C = len(lens), x.shape[1]
    state = torch.zeros(S, C, dtype=torch.float64, device="cuda") if st.h0 is None else st.h0.double().clone()
    start, n = st.offsets[:-1], torch.tensor(lens, device="cuda")
    h, before = torch.zeros_like(x), torch.zeros_like(x)
    for t in range(max(lens)):
        who = (n > t).nonzero()[:, 0]
        at = start[who] + t
        before[at] = state[who]
        state[who] = a[at] * state[who] + b[at] * x[at]
        h[at] = state[who]
    if not grad:
        return [h, state]
    dx, dg, dh = torch.zeros_like(x), torch.zeros_like(x), st.dh.double()
    c = torch.zeros_like(state) if st.dlast is None else st.dlast.double().clone()
    for t in reversed(range(max(lens))):
        who = (n > t).nonzero()[:, 0]
        at = start[who] + t
        d = dh[at] + c[who]
        dx[at], dg[at], c[who] = b[at] * d, d * (before[at] - x[at]) * a[at] * b[at], a[at] * d
    return [dx, dg, c if st.h0 is not None else None]


def _exact_attend(st, grad):
    """User by user and head by head."""
    c = st.case
    qo, ko = st.q_offsets.tolist(), st.k_offsets.tolist()
    lk = [b - a for a, b in zip(ko[:-1], ko[1:])] if st.k_lengths is None else st.k_lengths.tolist()
    o = torch.zeros(st.q.shape, dtype=torch.float64, device="cuda")
    lse = torch.full(st.q.shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    dq, dk, dv = torch.zeros_like(o), torch.zeros(st.k.shape, dtype=torch.float64, device="cuda"), torch.zeros(st.k.shape, dtype=torch.float64, device="cuda")
    for u in range(c["users"]):
        rows, n = slice(qo[u], qo[u + 1]), torch.arange(ko[u], ko[u] + lk[u], device="cuda")
        if st.key_mask is not None:
            n = n[st.key_mask[n] != 0]
        if not len(n):
            continue
        for hd in range(c["heads"]):
            g = hd // (c["heads"] // c["kv_heads"])
            q, k, v = st.q[rows, hd].double(), st.k[n, g].double(), st.v[n, g].double()
            s = q @ k.T * st.scale
            l = torch.logsumexp(s, 1)
            p = torch.exp(s - l[:, None])
            o[rows, hd], lse[rows, hd] = p @ v, l
            if grad:
                do = st.dout[rows, hd].double()
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True)) * st.scale
                dq[rows, hd] = ds @ k
                dk[n, g] += ds.T @ q
                dv[n, g] += p.T @ do
    return [dq, dk, dv] if grad else [o, lse]


def exact(case, seed):
    call, st = case["call"], prepare(case, seed)
    if call in ("scan", "scan_grad"):
        return _exact_scan(st, call == "scan_grad")
    if call in ("attend", "attend_grad"):
        return _exact_attend(st, call == "attend_grad")
    if call == "scan_step":
        e = torch.exp(-st.gate.double())
        h = (st.state.double() + e * st.x.double()) / (1 + e)
        return [h, h]
    tok = st.tokens.long()
    if call == "embed":
        out = st.table.double()[tok.clamp(min=0)] * SCALE
        out[tok < 0] = 0
        return out
    order = torch.argsort(tok, stable=True)
    order = order[tok[order] >= 0]
    rows, counts = torch.unique_consecutive(tok[order], return_counts=True)
    total = torch.zeros(len(rows), case["dim"], dtype=torch.float64, device="cuda")
    total.index_add_(0, torch.repeat_interleave(torch.arange(len(rows), device="cuda"), counts), st.grad[order].double())
    full = torch.zeros(case["rows"] if case["form"] == "table" else st.out["capacity"], case["dim"], dtype=torch.float64, device="cuda")
    full[rows if case["form"] == "table" else torch.arange(len(rows), device="cuda")] = total * SCALE
    return full if case["form"] == "table" else [None, full, None]


# ---------------------------------------------------------------------------------------------- what a pass has to do
def _distinct(rows, zipf, tokens):
    """Expected number of distinct rows among so many tokens (the sum over ranks taken over a logarithmic grid)."""
    edge = np.unique(np.rint(np.exp(np.linspace(0.0, math.log(rows + 1), 400))))
    mid, n = np.sqrt(edge[:-1] * (edge[1:] - 1).clip(1)), np.diff(edge)
    p = mid ** -zipf
    return float((n * -np.expm1(-tokens * p / (n * p).sum())).sum())


def _mean_length(longest):
    return (max(1, longest // 8) + longest) / 2


def work(case):
    """Operands once, outputs once; the products of the attention (two forward, five backward), a few operations an element elsewhere."""
    s = 2.0 if case["dtype"] == "bf16" else 4.0
    if case["call"] in ("embed", "embed_grad"):
        n, D = case["tokens"], case["dim"]
        d = _distinct(case["rows"], case["zipf"], n * 63 / 64)
        if case["call"] == "embed":
            return {"bytes": n * 4 + d * D * 4 + n * D * s, "flops": float(n * D)}
        return {"bytes": n * 4 + n * D * s * 63 / 64 + d * (D * 8 if case["form"] == "table" else D * 4 + 8), "flops": float(n * D)}
    if case["call"] == "scan_step":
        n = case["users"] * case["channels"]
        return {"bytes": n * (3 * s + 8), "flops": 8.0 * n}
    if case["call"] in ("scan", "scan_grad"):
        n, states = case["users"] * _mean_length(case["longest"]) * case["channels"], case["users"] * case["channels"] * 4.0
        if case["call"] == "scan":
            return {"bytes": 3 * n * s + states * (1 + case["state"]), "flops": 8.0 * n}
        return {"bytes": 6 * n * s + 3 * states * case["state"], "flops": 14.0 * n}
    u, H, G, D = case["users"], case["heads"], case["kv_heads"], case["dim"]
    lq = case["queries"] if case["cache"] or case["queries"] == 1 else _mean_length(case["queries"])
    lk = _mean_length(case["keys"])
    pairs, nq, nk = u * H * lq * lk * (0.9 if case["mask"] else 1.0), u * lq * H * D * s, u * lk * G * D * s
    if case["call"] == "attend":
        return {"bytes": 2 * nq + 2 * nk + u * lq * H * 4, "flops": 4.0 * pairs * D}
    return {"bytes": 4 * nq + 4 * nk + u * lq * H * 4, "flops": 10.0 * pairs * D}
