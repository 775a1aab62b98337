"""gm_seq_glu and gm_seq_glu_grad against 64 bits, within what fp32 arithmetic (and bf16 operands) may be off, element by element."""
import pytest
import torch

from tests import block_ref as B
from tests import seq_ref as R

gpu = pytest.mark.gpu
DTYPES = pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
ACTS = ["silu", "gelu", "sigmoid", "relu"]


@pytest.fixture(scope="module")
def gm():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=512 << 20)
    yield g
    g.close()


def _inputs(n, K, N, dtype, seed):
    """On the GPU, and so are the references: products of 64 bits."""
    gen = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=gen)  # noqa: E731
    x, wg, wu, dy = r(n, K).to(dtype), (r(K, N) * 1.5 / K ** 0.5).to(dtype), (r(K, N) / K ** 0.5).to(dtype), (r(n, N) * 0.1).to(dtype)
    return [t.cuda() for t in (x, wg, wu, r(N), r(N), dy)]


def _check(got, want, names, what=""):
    for i, name in enumerate(names):
        R.within(got[i], want[i].cpu(), want[i + len(names)].cpu(), f"{name} {what}")


GRADS = ("dx", "dw_gate", "dw_up", "db_gate", "db_up")
# one row to many; widths that end inside tiles of 32, 64, 128 and 256; every size of tile in all three products; rows in pieces
SHAPES = [(1, 8, 8), (5, 16, 24), (64, 512, 1024), (130, 72, 40), (300, 264, 136), (33, 1000, 104), (2100, 40, 1024), (8200, 1000, 1000), (16_400, 1000, 200), (100_003, 16, 24),
          (1500, 200, 264), (257, 128, 512), (4097, 8, 8), (700, 256, 256), (40, 64, 1096), (90, 200, 520)]


@gpu
@DTYPES
@pytest.mark.parametrize("shape", range(len(SHAPES)), ids=["x".join(map(str, s)) for s in SHAPES])
def test_glu_and_gradient(gm, shape, dtype):
    n, K, N = SHAPES[shape]
    x, wg, wu, bg, bu, dy = _inputs(n, K, N, dtype, shape)
    for bias, name in ((True, ACTS[shape % 4]), (False, ACTS[(shape + 1) % 4])):
        b = (bg, bu) if bias else (None, None)
        want = B.glu(x, wg, wu, *b, name)
        got = gm.seq_glu(x, wg, wu, name, b_gate=b[0], b_up=b[1], keep=True)
        _check(got, want, ("y", "gate", "up"), name)
        assert torch.equal(gm.seq_glu(x, wg, wu, name, b_gate=b[0], b_up=b[1]), got[0])
        wgrad = B.glu_grad(dy, x, wg, wu, got[1], got[2], name)
        grads = gm.seq_glu_grad(dy, x, wg, wu, got[1], got[2], name, bias=bias)
        if bias:
            _check(grads, wgrad, GRADS, name)
        else:
            assert grads[3] is None and grads[4] is None
            _check(grads[:3], wgrad[:3] + wgrad[5:8], GRADS[:3], name)
        again = gm.seq_glu_grad(dy, x, wg, wu, got[1], got[2], name, bias=bias)
        assert all(a is None or torch.equal(a, c) for a, c in zip(grads, again))           # a fixed order


@gpu
@DTYPES
@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("shape", [(70, 40, 72), (2100, 136, 1032)])
def test_rows_that_lie_apart(gm, shape, name, dtype):
    """Weights as halves of one array, rows inside wider ones, outputs between other values that stay."""
    n, K, N = shape
    x, wg, wu, bg, bu, dy = _inputs(n, K, N, dtype, 5)
    w = torch.cat([wg, wu], 1)
    wide = torch.full((n, K + 16), float("nan"), dtype=dtype, device="cuda")
    wide[:, 8:8 + K] = x
    y, gate, up = gm.seq_glu(x, wg, wu, name, b_gate=bg, b_up=bu, keep=True)
    room = torch.full((n, N + 24), 7.0, dtype=dtype, device="cuda")
    y2 = gm.seq_glu(wide[:, 8:8 + K], w[:, :N], w[:, N:], name, b_gate=bg, b_up=bu, out=room[:, 16:16 + N])
    assert torch.equal(y2, y) and (room[:, :16] == 7).all() and (room[:, 16 + N:] == 7).all()
    kept = torch.cat([gate, up], 1)
    dwide = torch.full((n, N + 8), float("nan"), dtype=dtype, device="cuda")
    dwide[:, 8:] = dy
    out, dw = torch.full((n, K + 8), 7.0, dtype=dtype, device="cuda"), torch.full((K, 2 * N + 8), 7.0, dtype=dtype, device="cuda")
    want = gm.seq_glu_grad(dy, x, wg, wu, gate, up, name, bias=True)
    got = gm.seq_glu_grad(dwide[:, 8:], wide[:, 8:8 + K], w[:, :N], w[:, N:], kept[:, :N], kept[:, N:], name, bias=True, out=(out[:, 8:], dw[:, :N], dw[:, N + 8:]))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and (out[:, :8] == 7).all() and (dw[:, N:N + 8] == 7).all()


@gpu
@DTYPES
@pytest.mark.parametrize("name", ACTS)
def test_activations_far_out(gm, name, dtype):
    """Pre-activations from -120 to 120 and zero, through one row of weights; and NaN stays in its row."""
    g = torch.cat([torch.linspace(-120, 120, 255), torch.zeros(1)]).to(dtype).cuda()
    x = torch.zeros(40, 8, dtype=dtype, device="cuda")
    x[:, 0] = 1
    wg, wu = torch.zeros(8, 256, dtype=dtype, device="cuda"), torch.zeros(8, 256, dtype=dtype, device="cuda")
    wg[0], wu[0] = g, 2
    got = gm.seq_glu(x, wg, wu, name, keep=True)
    _check(got, B.glu(x, wg, wu, None, None, name), ("y", "gate", "up"))
    dy = torch.ones(40, 256, dtype=dtype, device="cuda")
    grads = gm.seq_glu_grad(dy, x, wg, wu, got[1], got[2], name, bias=True)
    _check(grads, B.glu_grad(dy, x, wg, wu, got[1], got[2], name), GRADS)
    x[7, 3] = float("nan")
    y = gm.seq_glu(x, wg, wu, name)
    assert torch.isnan(y[7]).all() and torch.equal(y[:7], got[0][:7]) and torch.equal(y[8:], got[0][8:])


@gpu
@DTYPES
def test_no_rows(gm, dtype):
    x, wg, wu, bg, bu, dy = _inputs(0, 16, 24, dtype, 1)
    y, gate, up = gm.seq_glu(x, wg, wu, keep=True)
    dx, *rest = gm.seq_glu_grad(dy, x, wg, wu, gate, up, bias=True)
    assert y.shape == (0, 24) and dx.shape == (0, 16) and all((t == 0).all() for t in rest)


@gpu
@pytest.mark.parametrize("name", ["silu", "gelu", "sigmoid"])
def test_gradient_against_differences(gm, name):
    """Central differences of the 64-bit definition along random directions: off by some 1e-9 of the value, the gradient by 1e-6 and what keeping g and u in fp32 costs."""
    x, wg, wu, bg, bu, dy = _inputs(9, 24, 32, torch.float32, 2)
    _, gate, up = gm.seq_glu(x, wg, wu, name, b_gate=bg, b_up=bu, keep=True)
    grads = gm.seq_glu_grad(dy, x, wg, wu, gate, up, name, bias=True)
    gen = torch.Generator().manual_seed(4)
    value = lambda x, wg, wu, bg, bu: float((B.glu(x, wg, wu, bg, bu, name)[0] * dy).sum())  # noqa: E731
    args = (x, wg, wu, bg, bu)
    for i, grad in enumerate(grads):
        for _ in range(3):
            way = torch.randn(args[i].shape, generator=gen, dtype=torch.float64).cuda()
            plus, minus = ([t.double() + (way * k if j == i else 0) for j, t in enumerate(args)] for k in (1e-5, -1e-5))
            want = (value(*plus) - value(*minus)) / 2e-5
            assert abs(float((grad.double() * way).sum()) - want) <= 1e-5 * float((grad.double().abs() * way.abs()).sum())


@gpu
@DTYPES
def test_captured_and_on_another_stream(gm, dtype):
    from paper_2401_04338_amd import GMeta
    stream = torch.cuda.Stream()
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20, stream=stream.cuda_stream)
    g.configure("wait", 0)
    x, wg, wu, bg, bu, dy = _inputs(3000, 200, 136, dtype, 7)

    def both(g):
        y, gate, up = g.seq_glu(x, wg, wu, b_gate=bg, b_up=bu, keep=True)
        return (y, gate, up, *g.seq_glu_grad(dy, x, wg, wu, gate, up, bias=True))
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        both(g)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = both(g)
    for i in range(4):
        torch.cuda.synchronize()
        x.mul_(1.25)
        wu.mul_(0.5)
        dy.neg_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, both(gm))), i
    with torch.cuda.stream(torch.cuda.Stream()):
        there = both(gm)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(there, out))
    g.close()


@gpu
def test_refusals(gm):
    from paper_2401_04338_amd import GMetaError
    x, wg, wu, bg, bu, dy = _inputs(10, 16, 24, torch.bfloat16, 1)
    y, gate, up = gm.seq_glu(x, wg, wu, keep=True)
    for call in (lambda: gm.seq_glu(x, wg, wu, "tanh"), lambda: gm.seq_glu(x.float(), wg, wu), lambda: gm.seq_glu(x, wg, wu[:8]), lambda: gm.seq_glu(x.half(), wg.half(), wu.half()),
                 lambda: gm.seq_glu(x, wg, wu, b_gate=bg[:23], b_up=bu), lambda: gm.seq_glu(x, wg.t(), wu.t()), lambda: gm.seq_glu(x[0], wg, wu),
                 lambda: gm.seq_glu(x, wg, wu, out=torch.empty_like(x)), lambda: gm.seq_glu_grad(dy[:9], x, wg, wu, gate, up), lambda: gm.seq_glu_grad(dy, x, wg, wu, gate, up.float())):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: gm.seq_glu(x, wg, wu, b_gate=bg), lambda: gm.seq_glu(x[:, :12], wg[:12], wu[:12]), lambda: gm.seq_glu(x, wg[:, :20], wu[:, :20]),
                 lambda: gm.seq_glu(torch.zeros(10 * 16 + 4, dtype=torch.bfloat16, device="cuda")[4:].view(10, 16), wg, wu),
                 lambda: gm.seq_glu(x[:1].expand(10, 16), wg, wu), lambda: gm.seq_glu(torch.zeros(10, 20, dtype=torch.bfloat16, device="cuda")[:, :16], wg, wu),
                 lambda: gm.seq_glu(x, wg, wu, b_gate=torch.zeros(25, device="cuda")[1:], b_up=bu)):
        with pytest.raises(GMetaError) as e:
            call()
        assert e.value.code == -1
    p, lib = x.data_ptr(), gm.lib
    many = lambda *sizes: lib.gm_seq_glu(gm._ctx, *sizes, *[p, 1 << 17] * 3, None, None, p, 1 << 17, None, 0, None, 0)  # noqa: E731
    assert many(1 << 31, 16, 16, 1, 0) == -3 and many((1 << 31) - 1, 65536, 65536, 1, 0) == -3 and many(4, 16, 65544, 1, 0) == -1 and many(4, 16, 16, 2, 0) == -1
    assert many(4, 16, 16, 1, 4) == -1 and many(-1, 16, 16, 1, 0) == -1
    assert lib.gm_seq_glu(gm._ctx, 4, 16, 16, 1, 0, p, 1 << 20, p, 16, p, 16, None, None, p, 16, None, 0, None, 0) == -1
    assert lib.gm_seq_glu(gm._ctx, 4, 16, 16, 1, 0, p, 16, p, 16, p, 16, None, None, p, 16, p, 16, None, 0) == -1
    small = GMeta_small(gm, 1 << 20)
    big = _inputs(5000, 64, 256, torch.float32, 3)
    with pytest.raises(GMetaError) as e:
        small.seq_glu_grad(big[5], big[0], big[1], big[2], big[5], big[5])
    assert e.value.code == -4 and "needs" in str(e.value)
    small.close()
    assert torch.equal(gm.seq_glu(x, wg, wu), y)


def GMeta_small(gm, room):
    return type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=room)


@gpu
@DTYPES
def test_workspace_of_the_largest_call_holds_every_smaller_one(gm, dtype):
    kind, size = int(dtype == torch.bfloat16), gm.lib.gm_seq_glu_grad_bytes
    for other in ((512, 1024), (8, 8), (2000, 200)):
        sizes = [size(gm._ctx, n, *other, kind) for n in (0, 1, 5, 63, 64, 500, 511, 512, 1023, 1024, 5000, 8191, 8192, 33_000, 10 ** 6)]
        assert sizes == sorted(sizes) and sizes[0] > 0
    widths = [8, 64, 96, 104, 184, 192, 200, 256, 264, 512, 520, 1024, 4096]
    for n in (1, 600, 40_000):
        for fixed in (8, 200, 1024):
            for sizes in ([size(gm._ctx, n, w, fixed, kind) for w in widths], [size(gm._ctx, n, fixed, w, kind) for w in widths]):
                assert sizes == sorted(sizes)
    assert size(gm._ctx, 4, 12 if kind else 6, 16, kind) == size(gm._ctx, -1, 16, 16, kind) == size(gm._ctx, 4, 16, 16, 2) == 0
    most = GMeta_small(gm, size(gm._ctx, 9000, 264, 264, kind) + 4096)
    for n, K, N in ((9000, 264, 264), (9000, 8, 8), (8999, 96, 264), (2048, 264, 8), (9000, 256, 256), (9000, 192, 184), (1, 264, 264)):
        x, wg, wu, _, _, dy = _inputs(n, K, N, dtype, 1)
        got, want = (g.seq_glu_grad(dy, x, wg, wu, dy, dy, bias=True) for g in (most, gm))
        assert all(torch.equal(a, b) for a, b in zip(got, want))
    most.close()


def test_null_contexts():
    from paper_2401_04338_amd.binding import load_library
    lib = load_library()
    assert lib.gm_seq_glu(None, 0, 8, 8, 0, 0, *[None, 8] * 3, None, None, *[None, 8] * 3) == -1
    assert lib.gm_seq_glu_grad(None, 0, 8, 8, 0, 0, *[None, 8] * 9, None, None) == -1
    assert lib.gm_seq_glu_grad_bytes(None, 4, 8, 8, 0) == 0


@pytest.mark.parametrize("name", ACTS)
def test_the_reference(name):
    """The reference of these tests against the library's derivative, on the CPU."""
    gen = torch.Generator().manual_seed(1)
    x, wg, wu, bg, bu = (torch.randn(*s, generator=gen, dtype=torch.float64).requires_grad_() for s in ((6, 8), (8, 16), (8, 16), (16,), (16,)))
    y, g, u, *_ = B.glu(x, wg, wu, bg, bu, name)
    f = {"silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu, "sigmoid": torch.sigmoid, "relu": torch.relu}[name]
    z = f(x @ wg + bg) * (x @ wu + bu)
    assert (y - z).abs().max() < 1e-12
    dy = torch.randn(6, 16, generator=gen, dtype=torch.float64)
    want = torch.autograd.grad((z * dy).sum(), (x, wg, wu, bg, bu))
    got = B.glu_grad(dy, x.detach(), wg.detach(), wu.detach(), g.detach(), u.detach(), name)[:5]
    assert all((a - b).abs().max() < 1e-12 for a, b in zip(got, want))


# t, of which the tail goes with at most the third power, is off by 3 u, the polynomial by 9 u of twice its value, the exponential and its products by 6 u; the exponent's three
# roundings are 1.5 g^2 u
TAIL = lambda g: (1.5 * g * g + 36) * R.U  # noqa: E731


@gpu
@DTYPES
def test_the_tail_of_gelu_keeps_its_digits(gm, dtype):
    """gelu(g) and its slope from -13 to 13, relative to their values, not to g: down to 8e-37.  A row of one weight and one of ones, so that g and u arrive as they are."""
    g = torch.linspace(-13, 13, 2048).to(dtype)
    wg, wu = torch.zeros(8, 2048, dtype=dtype), torch.zeros(8, 2048, dtype=dtype)
    wg[0], wu[0] = g, 1
    x = torch.zeros(1, 8, dtype=dtype)
    x[0, 0] = 1
    y, gate, up = gm.seq_glu(x.cuda(), wg.cuda(), wu.cuda(), "gelu", keep=True)
    assert torch.equal(gate[0].cpu(), g)
    g = g.double()
    phi, density = 0.5 * torch.erfc(-g / 2 ** 0.5), torch.exp(-g * g / 2) / (2 * torch.pi) ** 0.5
    value, slope = g * phi, phi + g * density
    rel, out = TAIL(g), R.UB * 1.01 if dtype == torch.bfloat16 else R.U
    assert ((y[0].cpu().double() - value).abs() <= (rel + out) * value.abs()).all()
    dy = torch.ones(1, 2048, dtype=dtype, device="cuda")
    db_gate, db_up = gm.seq_glu_grad(dy, x.cuda(), wg.cuda(), wu.cuda(), gate, up, "gelu", bias=True)[3:]
    assert ((db_up.cpu().double() - value).abs() <= (rel + R.U) * value.abs()).all()
    assert ((db_gate.cpu().double() - slope).abs() <= rel * (phi + (g * density).abs()) + 2 * R.U * slope.abs()).all()


@gpu
@pytest.mark.parametrize("n,K,N,name", [(70, 12, 20, "silu"), (130, 4, 4, "gelu"), (1, 4, 36, "sigmoid"), (2500, 132, 1028, "relu")])
def test_fp32_widths_of_16_bytes(gm, n, K, N, name):
    """Widths that four, and no more, elements divide."""
    x, wg, wu, bg, bu, dy = _inputs(n, K, N, torch.float32, N)
    got = gm.seq_glu(x, wg, wu, name, b_gate=bg, b_up=bu, keep=True)
    _check(got, B.glu(x, wg, wu, bg, bu, name), ("y", "gate", "up"))
    _check(gm.seq_glu_grad(dy, x, wg, wu, got[1], got[2], name, bias=True), B.glu_grad(dy, x, wg, wu, got[1], got[2], name), GRADS)
