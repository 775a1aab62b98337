"""gm_seq_scan, gm_seq_scan_grad and gm_seq_scan_step against the recurrence in 64 bits, within a running bound of fp32 rounding."""
import pytest
import torch

from tests import seq_ref as R

pytestmark = pytest.mark.gpu
LENGTHS = {"one": [1], "empty": [0], "two": [2, 0], "short": [5, 0, 1, 31, 32, 33, 63, 64, 65, 7], "mixed": [300, 0, 129, 1, 128], "long": [3000, 0, 1, 700],
           "very_long": [20_011], "many": [40] * 300}


@pytest.fixture(scope="module")
def gm():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20)
    yield g
    g.close()


def _offsets(lengths):
    return torch.tensor([0] + lengths).cumsum(0).cuda()


def _inputs(lengths, C, dtype, seed, state=True):
    gen = torch.Generator().manual_seed(seed)
    N = sum(lengths)
    x, g = torch.randn(N, C, generator=gen).to(dtype), (torch.randn(N, C, generator=gen) * 1.5 + 2).clamp(-12, 12).to(dtype)
    h0 = torch.randn(len(lengths), C, generator=gen) if state else None
    return x, g, h0, gen


def _cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


CASES = [(k, C) for k, C in [("one", 1), ("empty", 8), ("two", 64), ("short", 3), ("short", 64), ("short", 100), ("mixed", 32), ("mixed", 256), ("long", 20),
                             ("long", 64), ("long", 7), ("very_long", 33), ("very_long", 64), ("many", 256)]]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("kind,C", CASES, ids=[f"{k}-{c}" for k, c in CASES])
@pytest.mark.parametrize("state", [True, False], ids=["state", "zero"])
def test_scan_and_gradient(gm, kind, C, dtype, state):
    lengths = LENGTHS[kind]
    x, g, h0, gen = _inputs(lengths, C, dtype, C + len(lengths), state)
    N, longest = sum(lengths), max(lengths)
    off = _offsets(lengths)
    xc, gc, h0c = _cuda(x, g, h0)
    h, last = gm.seq_scan(xc, gc, off, longest, h0=h0c)
    want, want_last, bound, last_bound = R.scan(x, g, lengths, h0)
    R.within(h, want, bound + R.out_round(want, dtype), "h")
    R.within(last, want_last, last_bound + R.U * want_last.abs(), "last")
    dh = torch.randn(N, C, generator=gen).to(dtype)
    dlast = torch.randn(len(lengths), C, generator=gen) if state else None
    hc = h.cpu()
    dhc, dlc = _cuda(dh, dlast)
    dx, dg, dh0 = gm.seq_scan_grad(dhc, xc, gc, h, off, longest, h0=h0c, dlast=dlc)
    wx, wg, w0, ex, eg, e0 = R.scan_grad(dh, x, g, hc, lengths, h0, dlast)
    R.within(dx, wx, ex + R.out_round(wx, dtype), "dx")
    R.within(dg, wg, eg + R.out_round(wg, dtype), "dgate")
    if state:
        R.within(dh0, w0, e0 + R.U * w0.abs(), "dh0")
    else:
        assert dh0 is None
    # a longer `longest` than any sequence has, and inputs whose rows lie apart and begin anywhere
    both = torch.full((N, 2 * C + 5), float("nan"), dtype=dtype, device="cuda")
    both[:, 1:1 + C], both[:, 2 + C:2 + 2 * C] = xc, gc
    h2, last2 = gm.seq_scan(both[:, 1:1 + C], both[:, 2 + C:2 + 2 * C], off, longest + 1000, h0=h0c)
    R.within(h2, want, bound + R.out_round(want, dtype), "h, strided")
    R.within(last2, want_last, last_bound + R.U * want_last.abs(), "last, strided")
    dx2, dg2, _ = gm.seq_scan_grad(dhc, both[:, 1:1 + C], both[:, 2 + C:2 + 2 * C], h, off, longest + 1000, h0=h0c, dlast=dlc)
    R.within(dx2, wx, ex + R.out_round(wx, dtype), "dx, strided")
    R.within(dg2, wg, eg + R.out_round(wg, dtype), "dgate, strided")


@pytest.mark.parametrize("C", [5, 64])
def test_gradient_against_differences(gm, C):
    """Central differences of the 64-bit recurrence: step 1e-5, so off by some 1e-9 of the values; h is fp32 (1e-7)."""
    lengths = [4, 0, 9]
    x, g, h0, gen = _inputs(lengths, C, torch.float32, 3)
    dh, dlast = torch.randn(13, C, generator=gen), torch.randn(3, C, generator=gen)

    def value(x, g, h0):
        h, last, _, _ = R.scan(x, g, lengths, h0)
        return (h * dh).sum(0) + (last * dlast).sum(0)      # per channel: the channels do not mix
    off = _offsets(lengths)
    h, _ = gm.seq_scan(*_cuda(x, g), off, 9, h0=h0.cuda())
    got = gm.seq_scan_grad(*_cuda(dh, x, g), h, off, 9, h0=h0.cuda(), dlast=dlast.cuda())
    for i, t in enumerate((x, g, h0)):
        args = [x.double(), g.double(), h0.double()]
        want = torch.zeros_like(t, dtype=torch.float64)
        for r in range(len(t)):
            vals = []
            for sign in (1, -1):
                a = [y.clone() for y in args]
                a[i][r] += sign * 1e-5
                vals.append(value(*a))
            want[r] = (vals[0] - vals[1]) / 2e-5
        assert float((got[i].cpu().double() - want).abs().max()) <= 1e-5 * float(want.abs().max())


@pytest.mark.parametrize("kind", ["short", "long"])
def test_extreme_gates_and_nan_stay_where_they_are(gm, kind):
    lengths, C = LENGTHS[kind], 64
    x, g, h0, gen = _inputs(lengths, C, torch.float32, 9)
    inf = float("inf")
    g[::3, 0], g[:, 1], g[:, 2], g[::2, 3], g[1::2, 3] = 60.0, inf, -inf, 200.0, -200.0
    off = _offsets(lengths)
    h, last = gm.seq_scan(*_cuda(x, g), off, max(lengths), h0=h0.cuda())
    want, want_last, bound, _ = R.scan(x, g, lengths, h0)
    # (beyond |g| = 12 the exponential is off by |g| u relatively, where it is 1e-5 of the other term and less)
    R.within(h, want, 2 * bound + R.U * want.abs() + 1e-30, "h")
    assert torch.equal(h[:, 2].cpu(), x[:, 2])                       # a = 0: h = x
    at = 0
    for s, n in enumerate(lengths):                                  # a = 1: the state stays
        assert torch.equal(h[at:at + n, 1].cpu(), h0[s, 1].expand(n))
        at += n
    xn = x.clone()
    row = lengths[0] // 2
    xn[row, 5] = float("nan")
    hn, _ = gm.seq_scan(*_cuda(xn, g), off, max(lengths), h0=h0.cuda())
    bad = torch.zeros_like(h, dtype=torch.bool)
    bad[row:lengths[0], 5] = True
    assert torch.equal(torch.isnan(hn), bad) and torch.equal(hn[~bad], h[~bad])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("S,C", [(1, 1), (3, 5), (7, 64), (513, 100), (1, 256)])
def test_steps_are_the_scan(gm, S, C, dtype):
    T = 6
    x, g, h0, _ = _inputs([T] * S, C, dtype, S + C)
    state, hs = h0.cuda(), []
    xs, gs = x.view(S, T, C).cuda(), g.view(S, T, C).cuda()
    for t in range(T):
        hs.append(gm.seq_scan_step(xs[:, t], gs[:, t], state))
    want, want_last, bound, last_bound = R.scan(x, g, [T] * S, h0)
    R.within(torch.stack(hs, 1).reshape(S * T, C), want, bound + R.out_round(want, dtype), "h")
    R.within(state, want_last, last_bound + R.U * want_last.abs(), "state")
    # the serving form takes the place of one more row of the scan
    off = _offsets([T] * S)
    _, last = gm.seq_scan(x.cuda(), g.cuda(), off, T, h0=h0.cuda())
    R.within(last, want_last, last_bound + R.U * want_last.abs(), "last")


def test_refusals(gm):
    from paper_2401_04338_amd import GMetaError
    x = torch.randn(10, 8, device="cuda")
    for off, longest in (([0, 4, 3, 10], 10), ([1, 4, 10], 10), ([0, 4, 9], 10), ([0, 4, 11], 10), ([0, 4, 10], 5), ([0, -1, 10], 11)):
        o = torch.tensor(off, device="cuda")
        with pytest.raises(GMetaError) as e:
            gm.seq_scan(x, x, o, longest)
        assert e.value.code == -2, off
        with pytest.raises(GMetaError) as e:
            gm.seq_scan_grad(x, x, x, x, o, longest)
        assert e.value.code == -2, off
    ok = torch.tensor([0, 4, 10], device="cuda")
    gm.seq_scan(x, x, ok, 6)
    for call in (lambda: gm.seq_scan(x, x[:9], ok, 6), lambda: gm.seq_scan(x, x.bfloat16(), ok, 6), lambda: gm.seq_scan(x.half(), x.half(), ok, 6),
                 lambda: gm.seq_scan(x, x, ok.int(), 6), lambda: gm.seq_scan(x, x, ok, 6, h0=torch.zeros(3, 8, device="cuda")),
                 lambda: gm.seq_scan(x.t(), x.t(), ok, 6), lambda: gm.seq_scan_step(x, x, torch.zeros(10, 8, device="cuda", dtype=torch.bfloat16)),
                 lambda: gm.seq_scan_grad(x, x, x, x, ok, 6, dlast=torch.zeros(2, 7, device="cuda"))):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(GMetaError) as e:
        gm.seq_scan(x, x, ok, -1)
    assert e.value.code == -1
    none = torch.zeros(1, dtype=torch.int64, device="cuda")
    h, last = gm.seq_scan(x[:0], x[:0], none, 0)
    assert h.shape == (0, 8) and last.shape == (0, 8)
    assert gm.lib.gm_seq_scan_bytes(4, 40_000, 256, 1) > 0 and gm.lib.gm_seq_scan_bytes(4096, 40_000, 256, 1) == 0


def test_offsets_whose_difference_wraps(gm):
    """Neighbouring offsets of either end of 64 bits: their difference, taken as it comes, is a length of 1."""
    from paper_2401_04338_amd import GMetaError
    x = torch.randn(10, 8, device="cuda")
    top, low = 2 ** 63 - 1, -2 ** 63
    for off in ([0, top, low, 10], [0, top, low + 2, 10], [0, low, top, 10], [0, 4, top, low, 10]):
        o = torch.tensor(off, device="cuda")
        for call in (lambda: gm.seq_scan(x, x, o, 10), lambda: gm.seq_scan_grad(x, x, x, x, o, 10)):
            with pytest.raises(GMetaError) as e:
                call()
            assert e.value.code == -2, off
    ok = torch.tensor([0, 4, 10], device="cuda")
    assert torch.isfinite(gm.seq_scan(x, x, ok, 6)[0]).all()


def test_rows_that_no_sequence_may_hold(gm):
    """`longest` 0 beside rows, as any other bound that a sequence exceeds."""
    from paper_2401_04338_amd import GMetaError
    x, off = torch.randn(10, 8, device="cuda"), torch.tensor([0, 4, 10], device="cuda")
    for call in (lambda: gm.seq_scan(x, x, off, 0), lambda: gm.seq_scan_grad(x, x, x, x, off, 0)):
        with pytest.raises(GMetaError) as e:
            call()
        assert e.value.code == -2 and "longest" in str(e.value)
    none = torch.zeros(3, dtype=torch.int64, device="cuda")
    h0 = torch.randn(2, 8, device="cuda")
    assert torch.equal(gm.seq_scan(x[:0], x[:0], none, 0, h0=h0)[1], h0)


@pytest.mark.parametrize("S,C,dtype", [(100, 256, torch.bfloat16), (3, 64, torch.float32), (1, 256, torch.bfloat16)], ids=["100", "3", "1"])
def test_a_workspace_that_many_sequences_do_not_need_takes_few(gm, S, C, dtype):
    """gm_seq_scan_bytes is 0 for a large batch and not for a small one: a context without that memory runs the small one, too."""
    lengths = [512 - 3 * i for i in range(S)] if S > 3 else [6000] * S
    assert gm.lib.gm_seq_scan_bytes(4096, max(lengths), C, 1 if dtype == torch.bfloat16 else 0) == 0 < gm.lib.gm_seq_scan_bytes(S, max(lengths), C, 1 if dtype == torch.bfloat16 else 0)
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=1 << 20)     # (the least a context has)
    x, g, h0, gen = _inputs(lengths, C, dtype, S)
    off, longest = _offsets(lengths), max(lengths)
    xc, gc, h0c = _cuda(x, g, h0)
    h, last = small.seq_scan(xc, gc, off, longest, h0=h0c)
    want, want_last, bound, last_bound = R.scan(x, g, lengths, h0)
    R.within(h, want, bound + R.out_round(want, dtype), "h")
    R.within(last, want_last, last_bound + R.U * want_last.abs(), "last")
    dh, dlast = torch.randn(sum(lengths), C, generator=gen).to(dtype), torch.randn(S, C, generator=gen)
    dx, dg, dh0 = small.seq_scan_grad(dh.cuda(), xc, gc, h, off, longest, h0=h0c, dlast=dlast.cuda())
    wx, wg, w0, ex, eg, e0 = R.scan_grad(dh, x, g, h.cpu(), lengths, h0, dlast)
    R.within(dx, wx, ex + R.out_round(wx, dtype), "dx")
    R.within(dg, wg, eg + R.out_round(wg, dtype), "dgate")
    R.within(dh0, w0, e0 + R.U * w0.abs(), "dh0")
    small.close()
