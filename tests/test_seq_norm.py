"""gm_seq_norm and gm_seq_norm_grad against 64 bits, within what fp32 arithmetic may be off, element by element."""
import ctypes as C

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


# one row to many, one channel to more than registers hold, widths of 16, 8 and 4 bytes; more rows than the gradient's workgroups take at a time
SHAPES = [(1, 1), (1, 64), (3, 8), (2, 0x10000), (5, 100), (64, 256), (130, 845), (1000, 36), (7, 2049), (33, 4096), (9, 1028), (9, 4100), (5, 8192), (6, 16_392), (3000, 3000), (5000, 512), (4101, 7), (33_000, 24), (4099, 1030), (70, 2048)]


def _inputs(n, Ch, dtype, seed, residual, far=0.0):
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x = (r(n, Ch) * torch.exp(r(n, 1)) + far).to(dtype)
    return x, r(n, Ch).to(dtype) if residual else None, r(Ch), r(Ch), (r(n, Ch) * 0.1).to(dtype), gen


def _cuda(*ts):
    return [None if t is None else t.cuda() for t in ts]


def _lie_apart(t, room, before):
    """The same rows, apart from each other, beginning anywhere; and the array they lie in."""
    n, Ch = t.shape
    whole = torch.full((n, Ch + room), 7.0, dtype=t.dtype, device="cuda")
    part = whole[:, before:before + Ch]
    part.copy_(t)
    return part, whole


@gpu
@DTYPES
@pytest.mark.parametrize("residual", [False, True], ids=["plain", "residual"])
@pytest.mark.parametrize("shape", SHAPES, ids=[f"{n}x{c}" for n, c in SHAPES])
def test_norm_and_gradient(gm, shape, residual, dtype):
    n, Ch = shape
    x, r, w, b, dy, gen = _inputs(n, Ch, dtype, n + Ch, residual)
    xc, rc, wc, bc, dyc = _cuda(x, r, w, b, dy)
    want = B.norm(x, r, w, b, 1e-5)
    got = gm.seq_norm(xc, wc, bc, residual=rc)
    for i, name in enumerate(("y", "s", "stats")):
        R.within(got[i], want[i], want[i + 3], name)
    assert (got[1] is xc) == (r is None)
    s, stats = got[1], got[2]
    e = (torch.randn(n, Ch, generator=gen) * 0.1).to(dtype) if residual else None
    wgrad = B.norm_grad(dy, s.cpu(), stats.cpu(), w, e)
    grads = gm.seq_norm_grad(dyc, s, stats, wc, dsum=None if e is None else e.cuda())
    for i, name in enumerate(("ds", "dweight", "dbias")):
        R.within(grads[i], wgrad[i], wgrad[i + 3], name)
    again = gm.seq_norm_grad(dyc, s, stats, wc, dsum=None if e is None else e.cuda())
    assert all(torch.equal(a, c) for a, c in zip(grads, again))           # a fixed order
    # rows that lie apart, at strides and beginnings that 16, 8 and no more bytes than an element divide; what lies between the outputs' rows stays
    for room, before in ((8, 0), (16, 8), (5, 1), (4, 4)):
        xs, rs = _lie_apart(xc, room, before)[0], None if r is None else _lie_apart(rc, room, before)[0]
        out, whole = _lie_apart(torch.zeros_like(xc), room, before)
        y2, s2, st2 = gm.seq_norm(xs, wc, bc, residual=rs, out=out)
        for i, t in enumerate((y2, s2, st2)):
            R.within(t, want[i], want[i + 3], f"strided {room} {before}")
        gap = torch.ones(Ch + room, dtype=torch.bool)
        gap[before:before + Ch] = False
        assert (whole[:, gap] == 7).all()
        ds, whole = _lie_apart(torch.zeros_like(xc), room, before)
        g2 = gm.seq_norm_grad(_lie_apart(dyc, room, before)[0], _lie_apart(s, room, before)[0], stats, wc,
                              dsum=None if e is None else _lie_apart(e.cuda(), room, before)[0], out=ds)
        for i, t in enumerate(g2):
            R.within(t, wgrad[i], wgrad[i + 3], f"gradient, strided {room} {before}")
        assert (whole[:, gap] == 7).all()


@gpu
@DTYPES
def test_without_weight_or_bias_and_rows_far_from_zero(gm, dtype):
    """Rows whose mean is a thousand deviations: the sum of squares is of the differences from it; rows that are all the same: only eps is left."""
    for far in (0.0, 1000.0):
        x, _, w, b, dy, _ = _inputs(40, 256, dtype, 3, False, far)
        x[5] = 3.0
        for weight, bias in ((None, None), (w, None), (None, b)):
            want = B.norm(x, None, weight, bias, 1e-3)
            got = gm.seq_norm(x.cuda(), *_cuda(weight, bias), eps=1e-3)
            for i in range(3):
                R.within(got[i], want[i], want[i + 3], f"far {far} output {i}")
            wg = B.norm_grad(dy, x, got[2].cpu(), weight, None)
            g = gm.seq_norm_grad(dy.cuda(), x.cuda(), got[2], *_cuda(weight))
            for i in range(3):
                R.within(g[i], wg[i], wg[i + 3], f"far {far} gradient {i}")


@gpu
def test_no_rows_and_rows_of_nan(gm):
    x = torch.empty(0, 64, device="cuda")
    y, s, stats = gm.seq_norm(x)
    ds, dw, db = gm.seq_norm_grad(x, x, stats)
    assert y.shape == (0, 64) and stats.shape == (0, 2) and ds.shape == (0, 64) and (dw == 0).all() and (db == 0).all()
    x = torch.randn(70, 96, device="cuda")
    want = gm.seq_norm(x)[0]
    x[33, 5], x[40, 1] = float("nan"), float("inf")
    got = gm.seq_norm(x)[0]
    bad = torch.zeros(70, dtype=torch.bool, device="cuda")
    bad[33] = bad[40] = True
    assert torch.equal(got[~bad], want[~bad]) and torch.isnan(got[33]).all() and torch.isnan(got[40, 1])


@gpu
def test_gradient_against_differences(gm):
    """Central differences of the 64-bit definition along random directions: off by some 1e-9 of the value, the gradient by 1e-6."""
    x, r, w, b, dy, gen = _inputs(6, 50, torch.float32, 9, True)
    e = torch.randn(6, 50, generator=gen)
    _, s, stats = gm.seq_norm(x.cuda(), w.cuda(), b.cuda(), residual=r.cuda())
    ds, dw, db = gm.seq_norm_grad(dy.cuda(), s, stats, w.cuda(), dsum=e.cuda())

    def value(x, w, b):
        y, s, *_ = B.norm(x, r, w, b, 1e-5)
        return float((y * dy).sum() + (s * e).sum())
    for i, (grad, args) in enumerate(((ds, x), (dw, w), (db, b))):
        for _ in range(3):
            way = torch.randn(args.shape, generator=gen, dtype=torch.float64)
            plus, minus = ([t.double() + (way * k if j == i else 0) for j, t in enumerate((x, w, b))] for k in (1e-5, -1e-5))
            want = (value(*plus) - value(*minus)) / 2e-5
            assert abs(float((grad.cpu().double() * way).sum()) - want) <= 1e-5 * float((grad.cpu().double().abs() * way.abs()).sum())


@gpu
@DTYPES
def test_captured_and_on_another_stream(gm, dtype):
    """Calls of one graph, replayed with other inputs and eager calls of other sizes (which use the same workspace) between; and on a stream of torch's own."""
    from paper_2401_04338_amd import GMeta
    stream = torch.cuda.Stream()
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20, stream=stream.cuda_stream)
    g.configure("wait", 0)
    x, r, w, b, dy, _ = _inputs(9000, 200, dtype, 5, True)
    x, r, w, b, dy = _cuda(x, r, w, b, dy)

    def both(g):
        y, s, stats = g.seq_norm(x, w, b, residual=r)
        return (y, s, stats, *g.seq_norm_grad(dy, s, stats, w))
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = both(g)
    torch.cuda.synchronize()
    for i in range(4):
        x.mul_(1.25)
        dy.add_(0.125)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        want = both(gm)
        assert all(torch.equal(a, c) for a, c in zip(out, want)), i
        gm.seq_norm_grad(dy[:999], x[:999], want[2][:999])
    with torch.cuda.stream(torch.cuda.Stream()):
        there = both(gm)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(there, both(gm)))
    g.close()


@gpu
def test_refused(gm):
    x, w = torch.randn(4, 8, device="cuda"), torch.ones(8, device="cuda")
    _, s, stats = gm.seq_norm(x)
    for call in (lambda: gm.seq_norm(x.half()), lambda: gm.seq_norm(x.view(4, 2, 4)), lambda: gm.seq_norm(x.cpu()), lambda: gm.seq_norm(x, w[:7]),
                 lambda: gm.seq_norm(x, w.bfloat16()), lambda: gm.seq_norm(x, residual=x[:3]), lambda: gm.seq_norm(x, residual=x.bfloat16()), lambda: gm.seq_norm(x.t()),
                 lambda: gm.seq_norm(x, out=torch.empty(4, 9, device="cuda")), lambda: gm.seq_norm_grad(x, x, stats[:3]), lambda: gm.seq_norm_grad(x[:3], x, stats),
                 lambda: gm.seq_norm_grad(x, x, stats, w[:3]), lambda: gm.seq_norm_grad(x, x, stats, dsum=x.bfloat16())):
        with pytest.raises(ValueError):
            call()
    from paper_2401_04338_amd.binding import GMetaError
    for call in (lambda: gm.seq_norm(x, eps=-1.0), lambda: gm.seq_norm(x, eps=float("nan")), lambda: gm.seq_norm(x[:1].expand(4, 8))):
        with pytest.raises(GMetaError) as e:
            call()
        assert e.value.code == -1
    p, lib = x.data_ptr(), gm.lib
    for rc, args in ((-1, (-1, 8, 0)), (-1, (4, 0, 0)), (-1, (4, 65537, 0)), (-1, (4, 8, 2)), (-3, (1 << 31, 8, 0))):
        assert lib.gm_seq_norm(gm._ctx, *args, p, 1 << 20, None, 0, None, None, 1e-5, p, 1 << 20, None, 0, None) == rc
        assert lib.gm_seq_norm_grad(gm._ctx, *args, p, 1 << 20, p, 1 << 20, stats.data_ptr(), None, None, 0, p, 1 << 20, None, None) == rc
    assert lib.gm_seq_norm(gm._ctx, 4, 8, 0, None, 8, None, 0, None, None, 1e-5, p, 8, None, 0, None) == -1
    assert lib.gm_seq_norm(gm._ctx, 4, 8, 0, p, 7, None, 0, None, None, 1e-5, p, 8, None, 0, None) == -1
    assert lib.gm_seq_norm(gm._ctx, 4, 8, 0, p, 8, None, 0, None, None, 1e-5, p, 8, None, 0, stats.data_ptr() + 4) == -1
    assert lib.gm_seq_norm_grad(gm._ctx, 4, 8, 0, p, 8, p, 8, stats.data_ptr(), None, None, 0, p, 8, w.data_ptr(), None) == -1
    assert lib.gm_seq_norm_grad(gm._ctx, 4, 8, 0, p, 8, p, 8, None, None, None, 0, p, 8, None, None) == -1


@gpu
def test_workspace_of_the_gradient(gm):
    from paper_2401_04338_amd import GMeta
    from paper_2401_04338_amd.binding import GMetaError
    need = gm.lib.gm_seq_norm_grad_bytes(6000, 512)
    x, dy = torch.randn(6000, 512, device="cuda"), torch.randn(6000, 512, device="cuda")
    _, s, stats = gm.seq_norm(x)
    want = gm.seq_norm_grad(dy, s, stats)
    exact = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=need + 4096)
    for n, Ch in ((6000, 512), (5999, 512), (6000, 33), (1, 512), (4096, 511)):   # (no more rows and channels)
        a, d = x[:n, :Ch].contiguous(), dy[:n, :Ch].contiguous()
        st = exact.seq_norm(a)[2]
        g = exact.seq_norm_grad(d, a, st)
        if (n, Ch) == (6000, 512):
            assert all(torch.equal(p, q) for p, q in zip(g, want))
    exact.close()
    little = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=need // 2)
    with pytest.raises(GMetaError) as e:
        little.seq_norm_grad(dy, s, stats)
    assert e.value.code == -4
    little.close()


def test_sizes_and_null_contexts():
    """No GPU is asked for these."""
    from paper_2401_04338_amd.binding import load_library
    lib = load_library()
    assert lib.gm_seq_norm(None, 0, 8, 0, None, 8, None, 0, None, None, 1e-5, None, 8, None, 0, None) == -1
    assert lib.gm_seq_norm_grad(None, 0, 8, 0, None, 8, None, 8, None, None, None, 0, None, 8, None, None) == -1
    for n, Ch in ((-1, 8), (1 << 31, 8), (4, 0), (4, 65537)):
        assert lib.gm_seq_norm_grad_bytes(n, Ch) == 0
    sizes = [lib.gm_seq_norm_grad_bytes(n, 256) for n in (0, 1, 100, 4096, 1 << 20, (1 << 31) - 1)]
    assert sizes == sorted(sizes) and sizes[-1] == 1024 * 2 * 256 * 4


@gpu
def test_more_rows_than_a_launch_holds_along_one_dimension(gm):
    """2^25 rows and some, a wave each: workgroups in two dimensions.  Rows at both ends and in the middle against 64 bits; the gradient of the last ones."""
    n, Ch = (1 << 25) + 5, 264
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty(n, Ch, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)
    y, s, stats = gm.seq_norm(x)
    for rows in (slice(0, 9), slice((1 << 24) - 3, (1 << 24) + 3), slice(n - 9, n)):
        want = B.norm(x[rows].cpu(), None, None, None, 1e-5)
        R.within(y[rows], want[0], want[3], "y")
        R.within(stats[rows], want[2], want[5], "stats")
    dy = torch.zeros(1, Ch, dtype=torch.bfloat16, device="cuda").expand(n, Ch).contiguous()
    dy[-9:] = 1
    ds, dw, db = gm.seq_norm_grad(dy, s, stats, out=y)
    want = B.norm_grad(dy[-9:].cpu(), x[-9:].cpu(), stats[-9:].cpu(), None, None)
    R.within(ds[-9:], want[0], want[3], "ds")
    R.within(dw, want[1], want[4], "dweight")
    assert (db == 9).all() and (ds[:9] == 0).all()
