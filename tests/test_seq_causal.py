"""gm_seq_attend_causal and gm_seq_attend_causal_grad against 64 bits, within what fp32 arithmetic (and bf16 operands) may be off, element by element."""
import pytest
import torch

from tests import block_ref as B
from tests import seq_ref as R

gpu = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])


@pytest.fixture(scope="module")
def gm():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20)
    yield g
    g.close()


def _off(lens):
    return [0] + torch.tensor(lens).cumsum(0).tolist() if lens else [0]


def _inputs(lq, lk, H, G, D, dtype, seed, mask):
    """mask: a quarter of the keys, among them the first of every sequence, and all of the last one's; masked rows hold rubbish, and so do the queries that see
    nothing but masked ones."""
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(sum(n), h, D, generator=gen).to(dtype) for n, h in ((lq, H), (lk, G), (lk, G)))
    m = None
    if mask:
        m = (torch.rand(sum(lk), generator=gen) < 0.75).to(torch.uint8)
        qo, ko = _off(lq), _off(lk)
        for s, n in enumerate(lk):
            m[ko[s]:ko[s] + min(n, 5 + 31 * s)] = 0
        m[ko[-2]:] = 0
        k[m == 0], v[m == 0] = float("nan"), float("inf")
        for s, n in enumerate(lk):
            on = m[ko[s]:ko[s + 1]].nonzero()
            first = int(on[0]) if len(on) else n
            q[qo[s]:qo[s] + max(0, min(lq[s], first - (n - lq[s])))] = float("nan")
    return q, k, v, m, gen


def _clean(t, m, dtype):
    return t if m is None else torch.where((m == 0)[:, None, None], torch.zeros((), dtype=dtype), t)


# queries and keys per sequence, heads, key heads, head width: whole histories, newest rows over longer ones, more queries than keys; rows of a workgroup 32, 64 and 128;
# groups that blocks of 32 rows cut
SHAPES = [([1], [1], 1, 1, 8), ([3, 0, 7, 64, 130], [3, 0, 7, 64, 130], 2, 2, 32), ([5, 1, 31], [5, 300, 31], 8, 2, 64), ([129, 2, 33], [129, 2, 33], 1, 1, 40),
          ([20, 5, 70], [63, 200, 70], 4, 1, 128), ([257, 40], [257, 40], 2, 1, 64), ([150, 129, 4], [65, 33, 500], 2, 2, 64), ([96], [96], 3, 3, 24),
          ([9, 300], [1000, 300], 4, 4, 16), ([190, 7], [190, 77], 2, 1, 120), ([5], [0], 2, 2, 64), ([64, 65], [64, 65], 1, 1, 128), ([1], [4000], 4, 2, 64), ([31], [1500], 1, 1, 128),
          ([100, 45], [100, 45], 3, 1, 64), ([70, 33, 200], [100, 33, 90], 5, 1, 96), ([520], [520], 6, 2, 128)]


def _run(gm, q, k, v, m, qo, ko, scale, bounds, gbounds, dtype, do, what):
    args = dict(scale=scale, key_mask=None if m is None else m.cuda(), causal=True)
    dev = [t.cuda() for t in (q, k, v)] + [torch.tensor(qo).cuda(), torch.tensor(ko).cuda()]
    lk = [b - a for a, b in zip(ko[:-1], ko[1:])]
    kz, vz = _clean(k, m, dtype), _clean(v, m, dtype)
    wo, wl, eo, el = B.attend(torch.nan_to_num(q), kz, vz, qo, ko[:-1], lk, scale, m)
    o, lse = gm.seq_attend(*dev, *bounds, **args)
    R.within(o, wo, eo, "o " + what)
    R.within(lse, wl, el, "lse " + what)
    want = B.attend_grad(do, q, kz, vz, o.cpu(), lse.cpu(), qo, ko[:-1], lk, scale, m)
    runs = [gm.seq_attend_grad(do.cuda(), *dev[:3], o, lse, *dev[3:], *gbounds, **args) for _ in range(2)]
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(runs[0][i], want[i], want[i + 3], f"{name} {what}")
    assert all(torch.equal(a, b) for a, b in zip(*runs))           # a fixed order
    return o, lse, want


@gpu
@DTYPES
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_causal_attention_and_gradient(gm, shape, mask, dtype):
    lq, lk, H, G, D = SHAPES[shape]
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, dtype, shape, mask)
    qo, ko, scale = _off(lq), _off(lk), 1.3 / D ** 0.5
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)
    if mask:
        do[torch.isnan(q[:, 0, 0])] = float("-inf")                # (what comes back for rows that see nothing)
    _run(gm, q, k, v, m, qo, ko, scale, (max(lq), max(lk)), (max(lq), max(lk)), dtype, do, "")
    # the other ways that a workgroup's waves may lie: by bounds that ask for more workgroups; the keys in pieces

    def rows_for(blocks, waves):
        return max(max(lq), -(-blocks // (len(lq) * G)) * 32 * waves // (H // G))

    def keys_for(blocks, waves):
        return max(max(lk), -(-blocks // (len(lk) * G)) * 32 * waves)
    grad_keys = (max(lk), keys_for(280, 2), keys_for(800, 4))             # waves along the keys for dk and dv: 1; 2 (fp32 with few rows: 4); 4
    _run(gm, q, k, v, m, qo, ko, scale, (max(lq), max(lk)), (max(max(lq), 300), grad_keys[1]), dtype, do, "two waves along the keys")
    for i, (fwd, dq) in enumerate(((max(lq), max(lq)), (rows_for(600, 2), rows_for(100, 2)), (rows_for(520, 4), rows_for(300, 4)))):
        _run(gm, q, k, v, m, qo, ko, scale, (fwd, 8192), (dq, grad_keys[i]), dtype, do, f"rows {fwd}, {dq}, keys {grad_keys[i]}")
        _run(gm, q, k, v, m, qo, ko, scale, (fwd, max(lk)), (dq, grad_keys[(i + 1) % 3]), dtype, do, f"rows {fwd}, {dq}, keys {grad_keys[(i + 1) % 3]}")


@gpu
@DTYPES
@pytest.mark.parametrize("users,cap,queries,H,G,D", [(3, 50, 1, 4, 2, 64), (2, 3000, 16, 8, 2, 64), (1, 2000, 3, 2, 2, 128), (5, 130, 40, 2, 1, 32), (64, 300, 16, 8, 2, 64)])
def test_newest_rows_over_slots_of_a_cache(gm, users, cap, queries, H, G, D, dtype):
    """Every user has a slot of the cache, filled up to a length, the newest rows' keys among them; what lies behind it is rubbish.  One query a user: as without order."""
    gen = torch.Generator().manual_seed(cap)
    lk = ([cap, queries, queries + 1, cap // 2, 33] + [int(x) for x in torch.randint(0, cap + 1, (60,), generator=gen)])[:users]
    q, k, v = torch.randn(users * queries, H, D, generator=gen).to(dtype), *(torch.randn(users * cap, G, D, generator=gen).to(dtype) for _ in range(2))
    for u, n in enumerate(lk):
        k[u * cap + n:(u + 1) * cap] = float("nan")
        v[u * cap + n:(u + 1) * cap] = float("-inf")
    qo, starts = _off([queries] * users), [u * cap for u in range(users)]
    args = [t.cuda() for t in (q, k, v)] + [torch.tensor(qo).cuda(), torch.tensor(starts + [users * cap]).cuda(), queries, cap]
    o, lse = gm.seq_attend(*args, k_lengths=torch.tensor(lk).cuda(), causal=True)
    wo, wl, eo, el = B.attend(q, torch.nan_to_num(k), torch.nan_to_num(v, neginf=0.0), qo, starts, lk, D ** -0.5, None)
    R.within(o, wo, eo, "o")
    R.within(lse, wl, el, "lse")
    if queries == 1:
        assert all(torch.equal(a, b) for a, b in zip((o, lse), gm.seq_attend(*args, k_lengths=torch.tensor(lk).cuda())))


@gpu
@DTYPES
@pytest.mark.parametrize("D", [32, 64, 128])
def test_a_prefix_does_not_see_what_follows(gm, D, dtype):
    """The rows of a history's first half are, bit for bit or within two roundings, those of the half alone; and changing the last row changes no other one."""
    gen = torch.Generator().manual_seed(D)
    n, H, G = 200, 4, 2
    q, k, v = (torch.randn(n, h, D, generator=gen).to(dtype).cuda() for h in (H, G, G))
    off = torch.tensor([0, n], device="cuda")
    o, lse = gm.seq_attend(q, k, v, off, off, n, n, causal=True)
    k[-1], v[-1] = k[-1] * 3 + 1, v[-1] - 5
    o2, lse2 = gm.seq_attend(q, k, v, off, off, n, n, causal=True)
    assert torch.equal(o[:-1], o2[:-1]) and torch.equal(lse[:-1], lse2[:-1]) and not torch.equal(lse[-1], lse2[-1])
    do = torch.randn(n, H, D, generator=gen).to(dtype).cuda()
    do[100:] = 0
    grads = gm.seq_attend_grad(do, q, k, v, o2, lse2, off, off, n, n, causal=True)
    assert all((g[100:] == 0).all() for g in grads)


@gpu
def test_gradient_against_differences(gm):
    """Central differences of the 64-bit definition along random directions: off by some 1e-9 of the value."""
    lq, lk, H, G, D, scale = [3, 40], [50, 40], 4, 2, 16, 0.3
    q, k, v, _, gen = _inputs(lq, lk, H, G, D, torch.float32, 5, False)
    m = (torch.rand(sum(lk), generator=gen) < 0.8).to(torch.uint8)
    do = torch.randn(sum(lq), H, D, generator=gen)
    qo, ko = _off(lq), _off(lk)
    dev = [t.cuda() for t in (q, k, v)]
    offs = torch.tensor(qo).cuda(), torch.tensor(ko).cuda()
    o, lse = gm.seq_attend(*dev, *offs, 40, 50, scale=scale, key_mask=m.cuda(), causal=True)
    got = gm.seq_attend_grad(do.cuda(), *dev, o, lse, *offs, 40, 50, scale=scale, key_mask=m.cuda(), causal=True)
    value = lambda q, k, v: float((B.attend(q, k, v, qo, ko[:-1], lk, scale, m)[0] * do).sum())  # noqa: E731
    for i in range(3):
        for _ in range(3):
            way = torch.randn(got[i].shape, generator=gen, dtype=torch.float64)
            plus, minus = ([t.double() + (way * s if j == i else 0) for j, t in enumerate((q, k, v))] for s in (1e-5, -1e-5))
            want = (value(*plus) - value(*minus)) / 2e-5
            assert abs(float((got[i].cpu().double() * way).sum()) - want) <= 1e-4 * float((got[i].cpu().double() * way).norm())


@gpu
@DTYPES
def test_many_ragged_histories(gm, dtype):
    """More sequences than are put in order, and enough of them that the order is made."""
    gen = torch.Generator().manual_seed(1)
    for users, longest in ((300, 60), (40, 700)):
        lens = [int(x) for x in torch.randint(0, longest + 1, (users,), generator=gen)]
        q, k, v, m, _ = _inputs(lens, lens, 4, 2, 64, dtype, users, True)
        off = _off(lens)
        do = torch.randn(sum(lens), 4, 64, generator=gen).to(dtype)
        _run(gm, q, k, v, m, off, off, 0.125, (longest, longest), (longest, longest), dtype, do, f"{users}")


@gpu
def test_captured(gm):
    from paper_2401_04338_amd import GMeta
    stream = torch.cuda.Stream()
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20, stream=stream.cuda_stream)
    g.configure("wait", 0)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q, k, v, do = (torch.randn(700, h, 64, device="cuda", generator=gen).bfloat16() for h in (4, 2, 2, 4))
    off = torch.tensor([0, 300, 300, 700], device="cuda")

    def both(g):
        o, lse = g.seq_attend(q, k, v, off, off, 400, 400, causal=True)
        return (o, lse, *g.seq_attend_grad(do, q, k, v, o, lse, off, off, 400, 400, causal=True))
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = both(g)
    for i in range(4):
        torch.cuda.synchronize()
        q.mul_(1.25)
        do.mul_(0.5)
        off[1] = 100 + 50 * i
        torch.cuda.synchronize()
        if i == 2:
            off[1], off[2] = 310, 310
            torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = both(gm)
        assert all(torch.equal(a, b) for a, b in zip(out, want)), i
        torch.cuda.synchronize()
    g.wait()
    g.close()


@gpu
def test_refusals(gm):
    from paper_2401_04338_amd import GMetaError
    q, k = torch.randn(10, 4, 64, device="cuda"), torch.randn(20, 2, 64, device="cuda")
    qo, ko = torch.tensor([0, 4, 10], device="cuda"), torch.tensor([0, 20, 20], device="cuda")
    o, lse = gm.seq_attend(q, k, k, qo, ko, 6, 20, causal=True)
    top, low = 2 ** 63 - 1, -2 ** 63
    for a, b, lq, lk in (([0, 4, 9], [0, 20, 20], 6, 20), ([0, 4, 10], [0, 20, 20], 5, 20), ([0, 4, 10], [0, 20, 20], 6, 19), ([0, 4, 10], [1, 20, 20], 6, 20),
                         ([4, 0, 10], [0, 20, 20], 10, 20), ([0, top, 10], [0, 20, 20], 6, 20), ([0, 4, 10], [0, low, 20], 6, 20)):
        a, b = torch.tensor(a, device="cuda"), torch.tensor(b, device="cuda")
        for call in (lambda: gm.seq_attend(q, k, k, a, b, lq, lk, causal=True), lambda: gm.seq_attend_grad(q, q, k, k, o, lse, a, b, lq, lk, causal=True)):
            with pytest.raises(GMetaError) as e:
                call()
            assert e.value.code == -2
    for call in (lambda: gm.seq_attend(q[:, :3].contiguous(), k, k, qo, ko, 6, 20, causal=True), lambda: gm.seq_attend(q, k, k, qo, ko, 6, 20, scale=0.0, causal=True)):
        with pytest.raises(GMetaError) as e:
            call()
        assert e.value.code == -1
    assert torch.equal(gm.seq_attend(q, k, k, qo, ko, 6, 20, causal=True)[0], o)


def test_null_contexts():
    from paper_2401_04338_amd.binding import load_library
    lib = load_library()
    assert lib.gm_seq_attend_causal(None, None, None, None, *[None, 0] * 3, None, None, 0, None) == -1
    assert lib.gm_seq_attend_causal_grad(None, None, None, None, *[None, 0] * 5, None, None, *[None, 0] * 3) == -1


def test_the_oracle_of_whole_rows():
    """The reference of these tests against a loop over single rows, on the CPU."""
    q, k, v, m, _ = _inputs([6, 3], [4, 9], 2, 1, 8, torch.float32, 1, False)
    m = torch.tensor([0, 1, 1, 0] + [1, 0, 1, 1, 1, 1, 1, 0, 1])
    o, lse, *_ = B.attend(q, k, v, [0, 6, 9], [0, 4], [4, 9], 0.5, m)
    for s, (q0, nq, k0, nk) in enumerate(((0, 6, 0, 4), (6, 3, 4, 9))):
        for i in range(nq):
            keys = [k0 + j for j in range(nk) if j <= i + nk - nq and m[k0 + j]]
            for h in range(2):
                if not keys:
                    assert (o[q0 + i, h] == 0).all() and lse[q0 + i, h] == -float("inf")
                    continue
                sc = torch.tensor([float(q[q0 + i, h].double() @ k[j, 0].double()) * 0.5 for j in keys], dtype=torch.float64)
                assert abs(float(lse[q0 + i, h]) - float(torch.logsumexp(sc, 0))) < 1e-12
                assert (o[q0 + i, h] - torch.softmax(sc, 0) @ v[keys, 0].double()).abs().max() < 1e-12


@gpu
def test_workspace_of_new_rows_over_slots(gm):
    """33 to 64 new rows lie on two waves, and the keys of few users are cut into pieces: what gm_seq_attend_bytes says for many users holds fewer, too."""
    from tests.test_seq_attend import _sizes
    queries, keys, H, G, D = 16, 4096, 8, 2, 64
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=_sizes(gm, 200, queries, keys, H, G, D, 1) + 4096)
    gen = torch.Generator().manual_seed(1)
    for users, new in ((200, 16), (64, 16), (64, 9), (5, 16), (1, 13)):
        q, k, v = (torch.randn(n, h, D, generator=gen).bfloat16() for n, h in ((users * new, H), (users * keys, G), (users * keys, G)))
        args = torch.arange(users + 1, device="cuda") * new, torch.arange(users + 1, device="cuda") * keys, new, keys
        o, lse = small.seq_attend(q.cuda(), k.cuda(), v.cuda(), *args, causal=True)
        want = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), *args, causal=True)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    small.close()


@gpu
@DTYPES
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("lq,lk,H,G,D", [([0, 3, 200], [40, 0, 7], 4, 2, 64), ([0, 150], [300, 150], 2, 1, 128), ([90, 0], [1, 70], 3, 1, 32)])
def test_keys_without_queries_and_queries_without_keys(gm, lq, lk, H, G, D, mask, dtype):
    """Keys that no query sees have no gradient; of more queries than keys the first see nothing."""
    gen = torch.Generator().manual_seed(D)
    q, k, v, do = (torch.randn(sum(n), h, D, generator=gen).to(dtype) for n, h in ((lq, H), (lk, G), (lk, G), (lq, H)))
    m = (torch.rand(sum(lk), generator=gen) < 0.5).to(torch.uint8) if mask else None
    qo, ko = _off(lq), _off(lk)
    for longest in ((max(lq), max(lk)), (700, 4000)):
        o, lse, _ = _run(gm, q, k, v, m, qo, ko, 0.2, longest, longest, dtype, do, f"{longest}")
        for s, (n, nk) in enumerate(zip(lq, lk)):
            blind = slice(qo[s], qo[s] + max(0, n - nk))
            assert (o[blind] == 0).all() and (lse[blind] == -float("inf")).all()
