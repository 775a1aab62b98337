"""gm_seq_attend and gm_seq_attend_grad against 64 bits, within what fp32 arithmetic (and bf16 operands) may be off, element by element."""
import ctypes as C
import math

import pytest
import torch

from tests import seq_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def gm():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20)
    yield g
    g.close()


def _off(lens):
    return [0] + torch.tensor(lens).cumsum(0).tolist() if lens else [0]


def _inputs(lq, lk, H, G, D, dtype, seed, mask):
    gen = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(sum(n), h, D, generator=gen).to(dtype) for n, h in ((lq, H), (lk, G), (lk, G)))
    m = None
    if mask:
        m = (torch.rand(sum(lk), generator=gen) < 0.7).to(torch.uint8)
        ko = _off(lk)
        m[ko[-2]:] = 0                                   # a user none of whose events counts
        k[m == 0], v[m == 0] = float("nan"), float("inf")
    return q, k, v, m, gen


# queries and keys per sequence, heads, key heads, head width: rows of a workgroup 32, 64 and 128, tiles that end anywhere, empty sides
SHAPES = [([1], [1], 1, 1, 8), ([3, 0, 5, 1], [0, 7, 64, 130], 2, 2, 32), ([1, 1, 1], [5, 300, 31], 8, 2, 64), ([33, 2], [128, 129], 1, 1, 40),
          ([20, 5, 0], [63, 200, 9], 4, 1, 128), ([70, 1], [1, 257], 2, 1, 64), ([150, 129, 4], [65, 33, 500], 2, 2, 64), ([260], [96], 3, 3, 24),
          ([9, 17], [1000, 40], 4, 4, 16), ([130, 7], [190, 77], 2, 1, 120), ([5], [0], 2, 2, 64), ([64, 65], [32, 64], 1, 1, 128), ([1], [4000], 4, 2, 64), ([31], [1500], 1, 1, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attention_and_gradient(gm, shape, mask, dtype):
    lq, lk, H, G, D = SHAPES[shape]
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, dtype, shape, mask)
    qo, ko, scale = _off(lq), _off(lk), 1.3 / D ** 0.5
    args = dict(scale=scale, key_mask=None if m is None else m.cuda())
    qc, kc, vc, qoc, koc = q.cuda(), k.cuda(), v.cuda(), torch.tensor(qo).cuda(), torch.tensor(ko).cuda()
    o, lse = gm.seq_attend(qc, kc, vc, qoc, koc, max(lq), max(lk), **args)
    if m is not None:
        k, v = (torch.where((m == 0)[:, None, None], torch.zeros((), dtype=dtype), t) for t in (k, v))
    wo, wl, eo, el = R.attend(q, k, v, qo, ko[:-1], lk, scale, m)
    R.within(o, wo, eo, "o")
    R.within(lse, wl, el, "lse")
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)
    want = R.attend_grad(do, q, k, v, o.cpu(), lse.cpu(), qo, ko[:-1], lk, scale, m)
    got = gm.seq_attend_grad(do.cuda(), qc, kc, vc, o, lse, qoc, koc, max(lq), max(lk), **args)
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(got[i], want[i], want[i + 3], name)
    again = gm.seq_attend_grad(do.cuda(), qc, kc, vc, o, lse, qoc, koc, max(lq), max(lk), **args)
    assert all(torch.equal(a, b) for a, b in zip(got, again))           # a fixed order
    # longer bounds than the lengths, keys and values side by side in one array, queries that lie apart
    kv = torch.zeros(len(k), 2 * G, D, dtype=dtype, device="cuda")
    kv[:, :G], kv[:, G:] = kc, vc
    wide = torch.zeros(len(q), H + 1, D, dtype=dtype, device="cuda")
    wide[:, :H] = qc
    o2, lse2 = gm.seq_attend(wide[:, :H], kv[:, :G], kv[:, G:], qoc, koc, max(lq) + 40, max(lk) + 300, **args)
    R.within(o2, wo, eo, "o, strided")
    R.within(lse2, wl, el, "lse, strided")
    got = gm.seq_attend_grad(do.cuda(), wide[:, :H], kv[:, :G], kv[:, G:], o, lse, qoc, koc, max(lq) + 40, max(lk) + 300, **args)
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(got[i], want[i], want[i + 3], name + ", strided")


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("waves", [2, 4])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_waves_along_rows_and_keys(gm, shape, waves, mask, dtype):
    """How a workgroup's waves lie, and whether the sequences are put in order first, follows from the workgroups that the longest lengths ask for: with large
    bounds on the lengths the kernels for many rows run on these short sequences, too."""
    lq, lk, H, G, D = SHAPES[shape]
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, dtype, 100 + shape, mask)
    qo, ko, scale = _off(lq), _off(lk), 1.3 / D ** 0.5
    args = dict(scale=scale, key_mask=None if m is None else m.cuda())

    def rows_for(blocks):   # a bound on the queries that asks for that many workgroups of 32 * waves rows
        return max(max(lq), -(-blocks // (len(lq) * G)) * 32 * waves // (H // G))

    def keys_for(blocks):
        return max(max(lk), -(-blocks // (len(lk) * G)) * 32 * waves)

    qc, kc, vc, qoc, koc = q.cuda(), k.cuda(), v.cuda(), torch.tensor(qo).cuda(), torch.tensor(ko).cuda()
    if m is not None:
        k, v = (torch.where((m == 0)[:, None, None], torch.zeros((), dtype=dtype), t) for t in (k, v))
    wo, wl, eo, el = R.attend(q, k, v, qo, ko[:-1], lk, scale, m)
    for longest_k in (max(lk), 8192):
        o, lse = gm.seq_attend(qc, kc, vc, qoc, koc, rows_for(600 if waves == 2 else 520), longest_k, **args)
        R.within(o, wo, eo, "o")
        R.within(lse, wl, el, "lse")
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)
    want = R.attend_grad(do, q, k, v, o.cpu(), lse.cpu(), qo, ko[:-1], lk, scale, m)
    runs = [gm.seq_attend_grad(do.cuda(), qc, kc, vc, o, lse, qoc, koc, rows_for(100 if waves == 2 else 300), keys_for(60 if waves == 2 else 300), **args) for _ in range(2)]
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(runs[0][i], want[i], want[i + 3], name)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("users,cap,queries,H,G,D", [(3, 50, 1, 4, 2, 64), (2, 3000, 1, 8, 2, 64), (1, 2000, 3, 2, 2, 128), (5, 130, 40, 2, 1, 32)])
def test_slots_of_a_cache(gm, users, cap, queries, H, G, D, dtype):
    """Every user has a slot of the cache, filled up to a length; what lies behind it is rubbish."""
    gen = torch.Generator().manual_seed(cap)
    lk = [cap, 0, 1, cap // 2, 33][:users]
    q, k, v = torch.randn(users * queries, H, D, generator=gen).to(dtype), *(torch.randn(users * cap, G, D, generator=gen).to(dtype) for _ in range(2))
    for u, n in enumerate(lk):
        k[u * cap + n:(u + 1) * cap] = float("nan")
        v[u * cap + n:(u + 1) * cap] = float("-inf")
    qo, starts = _off([queries] * users), [u * cap for u in range(users)]
    o, lse = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), torch.tensor(qo).cuda(), torch.tensor(starts + [users * cap]).cuda(), queries, cap,
                           k_lengths=torch.tensor(lk).cuda())
    wo, wl, eo, el = R.attend(q, torch.nan_to_num(k), torch.nan_to_num(v, neginf=0.0), qo, starts, lk, D ** -0.5, None)
    R.within(o, wo, eo, "o")
    R.within(lse, wl, el, "lse")


def test_gradient_against_differences(gm):
    """Central differences of the 64-bit definition along random directions: off by some 1e-9 of the value."""
    lq, lk, H, G, D, scale = [3, 40], [50, 9], 4, 2, 16, 0.3
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, torch.float32, 5, False)
    m = (torch.rand(sum(lk), generator=gen) < 0.8).to(torch.uint8)
    do = torch.randn(sum(lq), H, D, generator=gen)
    qo, ko = _off(lq), _off(lk)
    dev = [t.cuda() for t in (q, k, v)]
    offs = torch.tensor(qo).cuda(), torch.tensor(ko).cuda()
    o, lse = gm.seq_attend(*dev, *offs, 40, 50, scale=scale, key_mask=m.cuda())
    got = gm.seq_attend_grad(do.cuda(), *dev, o, lse, *offs, 40, 50, scale=scale, key_mask=m.cuda())
    value = lambda q, k, v: float((R.attend(q, k, v, qo, ko[:-1], lk, scale, m)[0] * do).sum())  # noqa: E731
    for i in range(3):
        for _ in range(3):
            way = torch.randn(got[i].shape, generator=gen, dtype=torch.float64)
            plus, minus = ([t.double() + (way * s if j == i else 0) for j, t in enumerate((q, k, v))] for s in (1e-5, -1e-5))
            want = (value(*plus) - value(*minus)) / 2e-5
            assert abs(float((got[i].cpu().double() * way).sum()) - want) <= 1e-4 * float((got[i].cpu().double() * way).norm())


def test_large_scores(gm):
    """Scores of some thousands, of either sign: a softmax that is nearly a maximum, without overflow."""
    q, k, v, _, _ = _inputs([40], [100], 1, 1, 64, torch.float32, 2, False)
    q, k = q.mul_(30).round_(), k.mul_(30).round_()                      # (whole numbers: the products are exact in fp32)
    o, lse = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), torch.tensor([0, 40]).cuda(), torch.tensor([0, 100]).cuda(), 40, 100, scale=0.125)
    wo, wl, eo, el = R.attend(q, k, v, [0, 40], [0], [100], 0.125, None)
    R.within(o, wo, eo, "o")
    R.within(lse, wl, el, "lse")
    assert float(wl.max()) > 1000


def test_nan_rows_stay_where_they_are(gm):
    q, k, v, _, _ = _inputs([40, 7], [100, 20], 2, 1, 64, torch.bfloat16, 2, False)
    offs = torch.tensor([0, 40, 47]).cuda(), torch.tensor([0, 100, 120]).cuda()
    o, lse = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), *offs, 40, 100)
    q[5, 1] = float("nan")
    k[110] = float("nan")                                               # a key that counts, of the second user
    on, ln = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), *offs, 40, 100)
    bad = torch.zeros(47, 2, dtype=torch.bool)
    bad[5, 1], bad[40:] = True, True
    assert torch.equal(torch.isnan(ln).cpu(), bad) and torch.isnan(on.cpu()[bad]).all()
    assert torch.equal(on.cpu()[~bad], o.cpu()[~bad]) and torch.equal(ln.cpu()[~bad], lse.cpu()[~bad])


def test_places_beyond_32_bits(gm):
    """Rows of a cache more than 2^31 elements (and 2^32 bytes) behind its first."""
    ld, rows = 1 << 20, 2600
    big = torch.empty(rows * ld, dtype=torch.bfloat16, device="cuda")
    kv = big.as_strided((rows, 2, 64), (ld, 64, 1))
    kv.normal_()
    q = torch.randn(4, 2, 64, device="cuda").bfloat16()
    starts, lens = [rows - 300, 0], [300, 70]
    qo = torch.tensor([0, 2, 4], device="cuda")
    o, lse = gm.seq_attend(q, kv[:, :1], kv[:, 1:], qo, torch.tensor(starts + [rows], device="cuda"), 2, 300, k_lengths=torch.tensor(lens, device="cuda"))
    k = kv.cpu()
    wo, wl, eo, el = R.attend(q.cpu(), k[:, :1], k[:, 1:], [0, 2, 4], starts, lens, 0.125, None)
    R.within(o, wo, eo, "o")
    R.within(lse, wl, el, "lse")
    x = kv[:, 0]
    off = torch.tensor([0, rows], device="cuda")
    h, last = gm.seq_scan(x, kv[:, 1], off, rows)
    wh, wlast, b, lb = R.scan(k[:, 0], k[:, 1], [rows], None)
    R.within(h, wh, b + R.out_round(wh, torch.bfloat16), "h")
    tok = torch.randint(0, 9, (rows,), device="cuda").to(torch.int32)
    g = gm.seq_embed_grad(x, tok, 9)
    wr, ws, wb = R.embed_grad(k[:, 0], tok.cpu(), 9, 1.0)
    R.within(g["emb_grad"][:len(wr)], ws, wb, "embed_grad")
    del big


def test_refusals(gm):
    from paper_2401_04338_amd import GMetaError
    q, k = torch.randn(10, 4, 64, device="cuda"), torch.randn(20, 2, 64, device="cuda")
    qo, ko = torch.tensor([0, 4, 10], device="cuda"), torch.tensor([0, 20, 20], device="cuda")
    gm.seq_attend(q, k, k, qo, ko, 6, 20)
    bad_offsets = (([0, 4, 9], [0, 20, 20], 6, 20), ([0, 4, 10], [0, 20, 20], 5, 20), ([0, 4, 10], [0, 20, 20], 6, 19), ([0, 4, 10], [0, 20, 21], 6, 21),
                   ([0, 4, 10], [1, 20, 20], 6, 20), ([4, 0, 10], [0, 20, 20], 10, 20))
    o, lse = gm.seq_attend(q, k, k, qo, ko, 6, 20)
    for a, b, lq, lk in bad_offsets:
        a, b = torch.tensor(a, device="cuda"), torch.tensor(b, device="cuda")
        with pytest.raises(GMetaError) as e:
            gm.seq_attend(q, k, k, a, b, lq, lk)
        assert e.value.code == -2
        with pytest.raises(GMetaError) as e:
            gm.seq_attend_grad(q, q, k, k, o, lse, a, b, lq, lk)
        assert e.value.code == -2
    with pytest.raises(GMetaError) as e:
        gm.seq_attend(q, k, k, qo, ko, 6, 20, k_lengths=torch.tensor([20, 1], device="cuda"))
    assert e.value.code == -2
    assert torch.equal(gm.seq_attend(q, k, k, qo, ko, 6, 20)[0], o)                        # the next call is clean
    codes = (lambda: gm.seq_attend(q[..., :62].contiguous(), k[..., :62].contiguous(), k[..., :62].contiguous(), qo, ko, 6, 20),   # no multiple of 16 bytes
             lambda: gm.seq_attend(torch.cat([q, q, q], 2), torch.cat([k, k, k], 2), torch.cat([k, k, k], 2), qo, ko, 6, 20),      # too wide
             lambda: gm.seq_attend(q[:, :3].contiguous(), k, k, qo, ko, 6, 20),                                                    # 3 heads over 2
             lambda: gm.seq_attend(q, k, k, qo, ko, 6, 20, scale=0.0), lambda: gm.seq_attend(q, k, k, qo, ko, 6, 20, scale=float("inf")),
             lambda: gm.seq_attend(torch.randn(10 * 256 + 1, device="cuda")[1:].view(10, 4, 64), k, k, qo, ko, 6, 20),             # not aligned
             lambda: gm.seq_attend(q, k, k, qo, ko[:2].contiguous(), 6, 20), lambda: gm.seq_attend(q, k, k, qo, ko, -1, 20))
    for call in codes:
        with pytest.raises(GMetaError) as e:
            call()
        assert e.value.code == -1
    for call in (lambda: gm.seq_attend(q, k.bfloat16(), k, qo, ko, 6, 20), lambda: gm.seq_attend(q, k, k[:19], qo, ko, 6, 20),
                 lambda: gm.seq_attend(q, k, k, qo, ko, 6, 20, key_mask=torch.ones(20, device="cuda")), lambda: gm.seq_attend(q.half(), k.half(), k.half(), qo, ko, 6, 20),
                 lambda: gm.seq_attend(q.transpose(0, 1), k, k, qo, ko, 6, 20), lambda: gm.seq_attend_grad(q, q, k, k, o, lse[:9], qo, ko, 6, 20)):
        with pytest.raises(ValueError):
            call()
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=1 << 20)
    one, far = torch.tensor([0, 200], device="cuda"), torch.tensor([0, 60_000], device="cuda")
    big = torch.randn(60_000, 4, 64, device="cuda")
    with pytest.raises(GMetaError) as e:
        small.seq_attend(big[:200], big, big, one, far, 200, 60_000)
    assert e.value.code == -4 and "needs" in str(e.value)
    small.close()


def test_offsets_and_lengths_whose_sums_wrap(gm):
    """Offsets and lengths of either end of 64 bits: differences and sums, taken as they come, are lengths and ends like any other."""
    from paper_2401_04338_amd import GMetaError
    q, k = torch.randn(10, 4, 64, device="cuda"), torch.randn(20, 2, 64, device="cuda")
    top, low = 2 ** 63 - 1, -2 ** 63
    qo, ko = [0, 4, 7, 10], [0, 8, 9, 20]
    o, lse = gm.seq_attend(q, k, k, torch.tensor(qo).cuda(), torch.tensor(ko).cuda(), 4, 11)
    for a, b, n in (([0, top, low, 10], ko, None), (qo, [0, top, low, 20], None), ([0, top, low + 3, 10], ko, None), (qo, [0, low, top, 20], None),
                    (qo, [0, top, 9, 20], [3, 1, 2]), (qo, [0, top - 5, 9, 20], [3, 11, 2]), (qo, [0, 8, 9, 20], [3, top, 2]), (qo, [0, 8, 9, 20], [3, low, 2]),
                    (qo, [low, 8, 9, 20], [3, 1, 2]), (qo, [0, 8, 21, 20], [3, 1, 0])):
        a, b, n = (None if t is None else torch.tensor(t, device="cuda") for t in (a, b, n))
        with pytest.raises(GMetaError) as e:
            gm.seq_attend(q, k, k, a, b, 4, 11, k_lengths=n)
        assert e.value.code == -2
        if n is None:
            with pytest.raises(GMetaError) as e:
                gm.seq_attend_grad(q, q, k, k, o, lse, a, b, 4, 11)
            assert e.value.code == -2
    assert torch.equal(gm.seq_attend(q, k, k, torch.tensor(qo).cuda(), torch.tensor(ko).cuda(), 4, 11)[0], o)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("D", [32, 64, 128])
@pytest.mark.parametrize("waves", [1, 2, 4])
def test_queries_of_users_without_a_key_that_counts(gm, waves, D, dtype):
    """A user all of whose events are masked: o = 0, lse = -infinity and no gradient, whatever the user's queries (and what comes back for them) hold; nothing
    of it reaches anyone else."""
    lq, lk, H, G = [3, 40, 5], [70, 600, 33], 4, 2
    q, k, v, _, gen = _inputs(lq, lk, H, G, D, dtype, 11, False)
    m = (torch.rand(sum(lk), generator=gen) < 0.7).to(torch.uint8)
    m[70:670] = 0
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)
    dirty, ddirty = q.clone(), do.clone()
    dirty[3:43:3], dirty[4:43:3, 1, 5], ddirty[5:43], ddirty[3, 2] = float("nan"), float("inf"), float("-inf"), float("nan")
    offs, mc = (torch.tensor(_off(lq)).cuda(), torch.tensor(_off(lk)).cuda()), m.cuda()
    # bounds on the lengths that lay one, two or four waves along the rows (and along the keys for dk and dv)
    bounds = {1: ((40, 600), (40, 600)), 2: ((64 * 300, 600), (64 * 10, 64 * 10)), 4: ((128 * 300, 600), (128 * 60, 128 * 60))}[waves]
    runs = []
    for x, dx in ((q, do), (dirty, ddirty)):
        xc, kc, vc = x.cuda(), k.cuda(), v.cuda()
        o, lse = gm.seq_attend(xc, kc, vc, *offs, *bounds[0], key_mask=mc)
        long = gm.seq_attend(xc, kc, vc, *offs, bounds[0][0], 8192, key_mask=mc)             # the keys in pieces, where the rows are few
        runs.append([o, lse, *long, *gm.seq_attend_grad(dx.cuda(), xc, kc, vc, o, lse, *offs, *bounds[1], key_mask=mc)])
    for name, a, b in zip(("o", "lse", "o of pieces", "lse of pieces", "dq", "dk", "dv"), *runs):
        assert torch.equal(a, b), name
        assert name in ("dk", "dv") or (b[3:43] == (-float("inf") if "lse" in name else 0)).all(), name


def test_rows_that_no_sequence_may_hold(gm):
    """`longest` 0 beside rows: like any other bound that a sequence exceeds.  Slots of a cache that are all empty are no such thing."""
    from paper_2401_04338_amd import GMetaError
    q, k = torch.randn(10, 4, 64, device="cuda"), torch.randn(20, 2, 64, device="cuda")
    qo, ko = torch.tensor([0, 4, 10], device="cuda"), torch.tensor([0, 20, 20], device="cuda")
    o, lse = gm.seq_attend(q, k, k, qo, ko, 6, 20)
    for lq, lk in ((0, 20), (6, 0), (0, 0)):
        with pytest.raises(GMetaError) as e:
            gm.seq_attend(q, k, k, qo, ko, lq, lk)
        assert e.value.code == -2 and "longest" in str(e.value)
        with pytest.raises(GMetaError) as e:
            gm.seq_attend_grad(q, q, k, k, o, lse, qo, ko, lq, lk)
        assert e.value.code == -2 and "longest" in str(e.value)
    empty, el = gm.seq_attend(q, k, k, qo, ko, 6, 0, k_lengths=torch.zeros(2, dtype=torch.int64, device="cuda"))
    assert (empty == 0).all() and (el == -float("inf")).all()
    dq, dk, dv = gm.seq_attend_grad(q[:0], q[:0], k, k, o[:0], lse[:0], torch.zeros(3, dtype=torch.int64, device="cuda"), ko, 0, 20)
    assert dq.shape == (0, 4, 64) and (dk == 0).all() and (dv == 0).all()
    assert torch.equal(gm.seq_attend(q, k, k, qo, ko, 6, 20)[0], o)


def _sizes(gm, users, queries, keys, H, G, D, bf16, grad=0):
    from paper_2401_04338_amd.binding import gm_seq, gm_seq_heads
    qs, ks, hd = gm_seq(users, users * queries, queries, None, None), gm_seq(users, users * keys, keys, None, None), gm_seq_heads(H, G, D, bf16, 1.0)
    return gm.lib.gm_seq_attend_bytes(gm._ctx, C.byref(qs), C.byref(ks), C.byref(hd), grad)


@pytest.mark.parametrize("bf16", [0, 1], ids=["fp32", "bf16"])
@pytest.mark.parametrize("H,G,D", [(8, 2, 64), (4, 4, 32), (8, 1, 128), (3, 3, 40)])
def test_workspace_of_the_largest_call_holds_every_smaller_one(gm, H, G, D, bf16):
    """Fewer users, queries or keys never ask for more: the keys are cut into more pieces where there are fewer rows."""
    for grad in (0, 1):
        for queries in (1, 5, 33, 70, 512):
            for keys in (1, 300, 4096, 100_000):
                sizes = [_sizes(gm, u, queries, keys, H, G, D, bf16, grad) for u in (1, 2, 3, 7, 16, 31, 64, 100, 128, 129, 200, 256, 257, 600, 5000)]
                assert sizes == sorted(sizes) and sizes[0] > 0
        for users in (1, 3, 64, 257):
            sizes = [_sizes(gm, users, n, 5000, H, G, D, bf16, grad) for n in (1, 2, 8, 31, 32, 33, 64, 65, 128, 129, 400, 3000)]
            assert sizes == sorted(sizes)
            sizes = [_sizes(gm, users, 4, n, H, G, D, bf16, grad) for n in (1, 255, 256, 511, 512, 513, 3000, 20_000, 10 ** 6)]
            assert sizes == sorted(sizes)
    assert _sizes(gm, -1, 1, 1, H, G, D, bf16) == _sizes(gm, 1, 1, -1, H, G, D, bf16) == _sizes(gm, 1, 1, 1, H, 0, D, bf16) == _sizes(gm, 1, 1, 1, H, G, -8, bf16) == 0


def test_a_context_for_many_users_takes_fewer(gm):
    """256 users' single queries fill the device without pieces; 64 users' keys are cut into pieces, in the workspace that was asked for the 256."""
    queries, keys, H, G, D = 1, 4096, 64, 2, 128
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=_sizes(gm, 256, queries, keys, H, G, D, 1) + 4096)
    gen = torch.Generator().manual_seed(1)
    for users in (64, 5):
        q, k, v = (torch.randn(n, h, D, generator=gen).bfloat16() for n, h in ((users, H), (users * keys, G), (users * keys, G)))
        args = torch.arange(users + 1, device="cuda"), torch.arange(users + 1, device="cuda") * keys, 1, keys
        o, lse = small.seq_attend(q.cuda(), k.cuda(), v.cuda(), *args)
        want = gm.seq_attend(q.cuda(), k.cuda(), v.cuda(), *args)
        assert torch.equal(o, want[0]) and torch.equal(lse, want[1])
    small.close()


# Scores that climb along the keys: by more than the 2^8 that the running maximum lets pass, in some blocks of 32 keys and not in others, at other keys for other rows;
# some rows climb never, some fall, some climb within one block.
def _climbing(lq, lk, H, G, D, dtype, seed, mask):
    gen = torch.Generator().manual_seed(seed)
    q, k = torch.zeros(sum(lq), H, D), torch.zeros(sum(lk), G, D)
    v = torch.randn(sum(lk), G, D, generator=gen)
    for s in range(len(lk)):
        for g in range(G):
            n = lk[s]
            at = torch.arange(n)
            rise = torch.zeros(n, 4)
            rise[:, 0] = (at // 32) * 16.0                                   # at every block of 32
            rise[:, 1] = (at // 192) * 30.0                                  # seldom
            rise[:, 2] = -(at // 64) * 20.0                                  # falls
            rise[:, 3] = torch.where(at == n - 1, 60.0, 0.0)                 # the last key alone
            k[_off(lk)[s]:_off(lk)[s] + n, g, :4] = rise
    which = torch.randint(0, 5, (sum(lq), H), generator=gen)
    for i in range(4):
        q[..., i] = (which == i).float()                                     # (4: none of them)
    q[..., 4:], k[..., 4:] = torch.randn(sum(lq), H, D - 4, generator=gen).round() / 4, torch.randn(sum(lk), G, D - 4, generator=gen).round() / 4
    m = None
    if mask:
        m = (torch.rand(sum(lk), generator=gen) < 0.7).to(torch.uint8)
        for s in range(len(lk)):
            m[_off(lk)[s]:_off(lk)[s] + min(150, lk[s] // 2)] = 0            # the first blocks hold nothing
    return q.to(dtype), k.to(dtype), v.to(dtype), m, gen


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("D", [16, 64, 128])
@pytest.mark.parametrize("waves", [1, 2, 4])
def test_scores_that_climb(gm, waves, D, mask, dtype):
    lq, lk, H, G = [40, 7, 130], [700, 33, 450], 4, 2
    q, k, v, m, gen = _climbing(lq, lk, H, G, D, dtype, waves + D, mask)
    qo, ko, scale = _off(lq), _off(lk), 1.0
    rises = _rises(q, k, qo, ko, m)
    assert (rises > 8).sum() > 100 and (rises < 1).sum() > 100               # in powers of two, over what came before: most rows several times, many rows never
    args = dict(scale=scale, key_mask=None if m is None else m.cuda())
    qc, kc, vc, offs = q.cuda(), k.cuda(), v.cuda(), (torch.tensor(qo).cuda(), torch.tensor(ko).cuda())
    wo, wl, eo, el = R.attend(q, k, v, qo, ko[:-1], lk, scale, m)
    bound = {1: 130, 2: 64 * 300, 4: 128 * 300}[waves]
    for longest_k in (700, 8192):                                            # (the second: the keys in pieces, where the rows are few)
        o, lse = gm.seq_attend(qc, kc, vc, *offs, bound, longest_k, **args)
        R.within(o, wo, eo, "o")
        R.within(lse, wl, el, "lse")
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)
    want = R.attend_grad(do, q, k, v, o.cpu(), lse.cpu(), qo, ko[:-1], lk, scale, m)
    got = gm.seq_attend_grad(do.cuda(), qc, kc, vc, o, lse, *offs, {1: 130, 2: 64 * 10, 4: 128 * 60}[waves], {1: 700, 2: 700, 4: 128 * 60}[waves], **args)
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(got[i], want[i], want[i + 3], name)


def _rises(q, k, qo, ko, m):
    """Every row's largest rise over the maximum of the blocks of 32 keys before, in powers of two."""
    H, G = q.shape[1], k.shape[1]
    out = []
    for s in range(len(qo) - 1):
        for h in range(H):
            sc = q[qo[s]:qo[s + 1], h].double() @ k[ko[s]:ko[s + 1], h // (H // G)].double().T / math.log(2)
            if m is not None:
                sc[:, m[ko[s]:ko[s + 1]] == 0] = -math.inf
            tops = torch.stack([b.amax(1) for b in sc.split(32, 1)], 1).cummax(1).values
            step = (tops[:, 1:] - tops[:, :-1]).nan_to_num(0.0, posinf=0.0, neginf=0.0) if tops.shape[1] > 1 else tops[:, :1] * 0
            out.append(step.amax(1))
    return torch.cat(out)


# Groups of query heads that do not divide 32, and one larger: blocks of 32 rows begin and end inside a query.
GROUPS = [([33, 7, 1], [70, 129, 5], 3, 1, 64), ([50, 0, 11], [300, 40, 9], 10, 2, 128), ([9, 31], [200, 77], 12, 1, 40), ([5, 70, 1], [100, 33, 64], 40, 1, 64),
          ([13, 4], [130, 31], 80, 2, 32), ([1, 22], [500, 3], 7, 1, 128)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("mask", [False, True], ids=["all", "masked"])
@pytest.mark.parametrize("waves", [1, 2, 4])
@pytest.mark.parametrize("shape", range(len(GROUPS)))
def test_groups_that_blocks_cut(gm, shape, waves, mask, dtype):
    lq, lk, H, G, D = GROUPS[shape]
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, dtype, 300 + shape, mask)
    qo, ko, scale = _off(lq), _off(lk), 1.3 / D ** 0.5
    args = dict(scale=scale, key_mask=None if m is None else m.cuda())
    do = torch.randn(sum(lq), H, D, generator=gen).to(dtype)

    def apart(t, more):   # rows that lie apart
        wide = torch.full((len(t), t.shape[1] + more, D), 7.0, dtype=dtype, device="cuda")
        wide[:, :t.shape[1]] = t.cuda()
        return wide[:, :t.shape[1]]
    qc, kc, vc, dc, offs = apart(q, 1), apart(k, 2), apart(v, 1), apart(do, 3), (torch.tensor(qo).cuda(), torch.tensor(ko).cuda())
    if m is not None:
        k, v = (torch.where((m == 0)[:, None, None], torch.zeros((), dtype=dtype), t) for t in (k, v))
    wo, wl, eo, el = R.attend(q, k, v, qo, ko[:-1], lk, scale, m)
    pairs = len(lq) * G
    rows = lambda blocks: max(max(lq), -(-(-(-blocks // pairs) * 32 * waves) // (H // G)))  # noqa: E731   (a bound that asks for so many workgroups)
    for longest_k in (max(lk), 8192):
        o, lse = gm.seq_attend(qc, kc, vc, *offs, max(lq) if waves == 1 else rows(600), longest_k, **args)
        R.within(o, wo, eo, "o")
        R.within(lse, wl, el, "lse")
    want = R.attend_grad(do, q, k, v, o.cpu(), lse.cpu(), qo, ko[:-1], lk, scale, m)
    bounds = {1: (max(lq), max(lk)), 2: (rows(100), max(lk)), 4: (rows(300), max(max(lk), -(-300 // pairs) * 128))}[waves]
    runs = [gm.seq_attend_grad(dc, qc, kc, vc, o, lse, *offs, *bounds, **args) for _ in range(2)]
    for i, name in enumerate(("dq", "dk", "dv")):
        R.within(runs[0][i], want[i], want[i + 3], name)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("waves", [1, 2, 4])
@pytest.mark.parametrize("D", [32, 64, 120])
def test_outputs_that_lie_apart(gm, D, waves, dtype):
    """Rows of outputs between rows of something else: the values of outputs that lie side by side, and nothing else is written."""
    lq, lk, H, G = [40, 0, 133], [70, 5, 600], 4, 2
    q, k, v, m, gen = _inputs(lq, lk, H, G, D, dtype, 5, True)
    qc, kc, vc, mc, do = q.cuda(), k.cuda(), v.cuda(), m.cuda(), torch.randn(sum(lq), H, D, generator=gen).to(dtype).cuda()
    offs = torch.tensor(_off(lq)).cuda(), torch.tensor(_off(lk)).cuda()

    def apart(n, heads):
        wide = torch.full((n, heads + 3, D), 5.0, dtype=dtype, device="cuda")
        return wide, wide[:, 1:1 + heads]
    for bounds in ((133, 600), (133, 8192)) if waves == 1 else ((32 * waves * 300, 600),):
        wide, view = apart(sum(lq), H)
        o, lse = gm.seq_attend(qc, kc, vc, *offs, *bounds, key_mask=mc)
        got, lse2 = gm.seq_attend(qc, kc, vc, *offs, *bounds, key_mask=mc, out=view)
        assert got is view and torch.equal(view, o) and torch.equal(lse, lse2)
        assert (wide[:, :1] == 5).all() and (wide[:, 1 + H:] == 5).all()
    bounds = {1: (133, 600), 2: (64 * 20, 600), 4: (128 * 60, 128 * 60)}[waves]
    want = gm.seq_attend_grad(do, qc, kc, vc, o, lse, *offs, *bounds, key_mask=mc)
    wides = [apart(sum(lq), H), apart(sum(lk), G), apart(sum(lk), G)]
    got = gm.seq_attend_grad(do, qc, kc, vc, o, lse, *offs, *bounds, key_mask=mc, out=[w[1] for w in wides])
    for (wide, view), g, x in zip(wides, got, want):
        assert g is view and torch.equal(view, x)
        assert (wide[:, :1] == 5).all() and (wide[:, 1 + x.shape[1]:] == 5).all()


def test_lengths_within_a_tile_of_31_bits(gm):
    """Places inside a sequence are 32-bit numbers, and so are those of the tile that goes beyond its end: the last lengths below 2^31 are refused."""
    from paper_2401_04338_amd import GMetaError
    q, off = torch.randn(4, 1, 8, device="cuda"), torch.tensor([0, 4], device="cuda")
    o, lse = gm.seq_attend(q, q, q, off, off, 4, 4)
    for lq, lk in ((4, 2 ** 31 - 100), (2 ** 31 - 100, 4), (4, 2 ** 31 - 1), (2 ** 31 - 1, 4)):
        for call in (lambda: gm.seq_attend(q, q, q, off, off, lq, lk), lambda: gm.seq_attend_grad(q, q, q, q, o, lse, off, off, lq, lk)):
            with pytest.raises(GMetaError) as e:
                call()
            assert e.value.code == -3
    far = gm.seq_attend(q, q, q, off, off, 4, 2 ** 31 - 300)
    assert torch.allclose(far[0], o, rtol=1e-5, atol=1e-6)
