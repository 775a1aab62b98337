"""gm_seq_embed and gm_seq_embed_grad against 64 bits: integers exactly, floats within what fp32 sums may be off."""
import ctypes as C

import pytest
import torch

from tests import seq_ref as R


def test_workspace_is_host_only_and_grows():
    from paper_2401_04338_amd import load_library
    lib = load_library()
    a, b, c = (lib.gm_seq_embed_grad_bytes(n, d) for n, d in ((1000, 16), (100_000, 16), (100_000, 64)))
    assert 0 < a < b < c
    assert lib.gm_seq_embed_grad_bytes(-1, 16) == 0 and lib.gm_seq_embed_grad_bytes(10, 0) == 0
    assert lib.gm_seq_embed(None, 0, None, 1, 4, None, 1.0, 0, None, 4) == -1       # no context
    assert lib.gm_wait(None) == -1


@pytest.fixture(scope="module")
def gm():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20)
    yield g
    g.close()


def _tokens(kind, n, rows, gen):
    if kind == "one":
        return torch.full((n,), rows - 1, dtype=torch.int32)
    if kind == "padding":
        return torch.full((n,), -1, dtype=torch.int32)
    if kind == "distinct":
        return (torch.randperm(rows, generator=gen)[:n]).to(torch.int32)
    t = (torch.rand(n, generator=gen) ** 4 * rows).long().clamp_(max=rows - 1)     # skewed, some padding
    return torch.where(torch.rand(n, generator=gen) < 0.1, -1, t).to(torch.int32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("n,dim", [(0, 8), (1, 1), (5, 3), (257, 4), (100, 36), (4099, 64), (63, 100), (33, 128), (7, 600), (3, 5000)])
def test_lookup(gm, n, dim, dtype):
    gen = torch.Generator().manual_seed(n * 1000 + dim)
    table, tokens = torch.randn(97, dim, generator=gen), _tokens("skewed", n, 97, gen)
    want = torch.where((tokens >= 0)[:, None], table[tokens.clamp(min=0).long()] * 0.3, torch.zeros(())).to(dtype)
    table[5] = float("nan")
    want[tokens == 5] = float("nan")
    got = gm.seq_embed(table.cuda(), tokens.cuda(), 0.3, dtype=dtype)
    assert got.dtype == dtype and torch.equal(torch.nan_to_num(got.cpu().float(), nan=77.0), torch.nan_to_num(want.float(), nan=77.0))   # one product, one rounding
    # rows that lie apart, and rows that begin between 16-byte units
    for pad, shift in ((24, 8), (7, 3)):
        wide = torch.full((n, dim + pad), 5.0, dtype=dtype, device="cuda")
        gm.seq_embed(table.cuda(), tokens.cuda(), 0.3, dtype=dtype, out=wide[:, shift:shift + dim])
        assert torch.equal(torch.nan_to_num(wide[:, shift:shift + dim].float(), nan=77.0), torch.nan_to_num(got.float(), nan=77.0))
        assert (wide[:, :shift] == 5).all() and (wide[:, shift + dim:] == 5).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("kind,n,rows,dim", [("skewed", 1, 1, 1), ("skewed", 31, 50, 3), ("skewed", 33, 5, 4), ("skewed", 3000, 97, 36), ("one", 20_000, 65, 64),
                                             ("one", 32, 2, 8), ("one", 1025, 4096, 16), ("padding", 500, 9, 16), ("distinct", 4096, 4096, 100), ("skewed", 5000, 2, 128),
                                             ("skewed", 400, 31, 600), ("skewed", 100_000, 70_000, 32), ("skewed", 0, 7, 8), ("skewed", 60, 11, 2500)])
def test_gradient(gm, kind, n, rows, dim, dtype):
    gen = torch.Generator().manual_seed(n + rows + dim)
    tokens, grad = _tokens(kind, n, rows, gen), torch.randn(n, dim, generator=gen).to(dtype)
    grad[tokens == -1] = float("nan")                       # what padding's rows hold has no influence
    clean = torch.where((tokens == -1)[:, None], torch.zeros((), dtype=dtype), grad)
    want_rows, want, bound = R.embed_grad(clean, tokens, rows, -0.7)
    runs = []
    for _ in range(2):
        out = gm.seq_embed_grad(grad.cuda(), tokens.cuda(), rows, -0.7)
        k = int(out["n_emb_rows"])
        assert k == len(want_rows) and torch.equal(out["emb_rows"][:k].cpu(), want_rows)
        R.within(out["emb_grad"][:k], want, bound, "list")
        runs.append(out["emb_grad"][:k].clone())
    assert torch.equal(*runs)                               # a fixed order
    table = torch.randn(rows, dim, generator=gen)
    full, full_bound = table.double().clone(), torch.zeros(rows, dim, dtype=torch.float64)
    full[want_rows] += want
    full_bound[want_rows] = bound + R.U * full[want_rows].abs()
    got = gm.seq_embed_grad(grad.cuda(), tokens.cuda(), rows, -0.7, table=table.cuda())
    R.within(got, full, full_bound, "table")
    # gradient rows that lie apart
    wide = torch.zeros(n, dim + 9, dtype=dtype, device="cuda")
    wide[:, 1:1 + dim] = grad.cuda()
    out = gm.seq_embed_grad(wide[:, 1:1 + dim], tokens.cuda(), rows, -0.7)
    R.within(out["emb_grad"][:k], want, bound, "strided")


@pytest.mark.gpu
@pytest.mark.parametrize("n", [63, 65, 1024, 1025, 8191, 8192, 8193, 131_073, 524_288, 524_289])
@pytest.mark.parametrize("rows", [1, 255, 256, 70_000, 1 << 24])
def test_lengths_where_the_sort_changes(gm, n, rows):
    """Rows, their number and their sums at the lengths where one way to sort ends and the next begins: whole numbers, whose fp32 sums below 2^24 are exact."""
    gen = torch.Generator().manual_seed(n + rows)
    tokens = _tokens("skewed", n, rows, gen)
    grad = torch.ones(n, 1)
    out = gm.seq_embed_grad(grad.cuda(), tokens.cuda(), rows)
    want, counts = torch.unique(tokens[tokens >= 0], return_counts=True)
    k = int(out["n_emb_rows"])
    assert k == len(want) and torch.equal(out["emb_rows"][:k].cpu(), want.to(torch.int64))
    assert torch.equal(out["emb_grad"][:k, 0].cpu(), counts.to(torch.float32))      # whole numbers below 2^24: exact in any order
    grad = torch.arange(n, dtype=torch.float32)[:, None] % 4096                      # whose positions they are
    out = gm.seq_embed_grad(grad.cuda(), tokens.cuda(), rows)
    sums = torch.zeros(rows, dtype=torch.float64).index_add_(0, tokens[tokens >= 0].long(), grad[tokens >= 0, 0].double())
    few = sums[want.long()] < 2 ** 24
    assert torch.equal(out["emb_grad"][:k, 0].cpu().double()[few], sums[want.long()][few])


@pytest.mark.gpu
def test_refusals_and_what_the_device_finds(gm):
    from paper_2401_04338_amd import GMetaError
    table, ok = torch.randn(50, 8, device="cuda"), torch.zeros(10, dtype=torch.int32, device="cuda")
    for bad in (50, -2, 2 ** 31 - 1, -2 ** 31):
        t = ok.clone()
        t[3] = bad
        with pytest.raises(GMetaError) as e:
            gm.seq_embed(table, t)
        assert e.value.code == -2
        with pytest.raises(GMetaError) as e:
            gm.seq_embed_grad(torch.ones(10, 8, device="cuda"), t, 50)
        assert e.value.code == -2
    assert torch.equal(gm.seq_embed(table, ok), table[ok.long()])      # the next call is clean
    with pytest.raises(GMetaError) as e:
        gm.seq_embed_grad(torch.ones(10, 8, device="cuda"), torch.arange(10, dtype=torch.int32, device="cuda"), 50, emb_rows_capacity=9)
    assert e.value.code == -3
    # enqueued only: the error comes with the wait, once
    gm.configure("wait", 0)
    t = ok.clone()
    t[0] = 77
    gm.seq_embed(table, t)
    with pytest.raises(GMetaError) as e:
        gm.wait()
    assert e.value.code == -2
    gm.wait()
    gm.configure("wait", 1)
    for call in (lambda: gm.seq_embed(table, ok.long()), lambda: gm.seq_embed(table.double(), ok), lambda: gm.seq_embed(table.cpu(), ok),
                 lambda: gm.seq_embed(table, ok, dtype=torch.float16), lambda: gm.seq_embed(table, ok, out=torch.empty(9, 8, device="cuda")),
                 lambda: gm.seq_embed_grad(torch.ones(9, 8, device="cuda"), ok, 50),
                 lambda: gm.seq_embed_grad(torch.ones(10, 8, device="cuda"), ok, 50, table=table[:49])):
        with pytest.raises(ValueError):
            call()
    for args in ((0, 8, 1.0), (2 ** 31 - 1, 8, 1.0)):
        rc = gm.lib.gm_seq_embed(gm._ctx, 10, C.c_void_p(ok.data_ptr()), args[0], args[1], C.c_void_p(table.data_ptr()), args[2], 0, C.c_void_p(table.data_ptr()), 8)
        assert rc == -1
    with pytest.raises(GMetaError) as e:
        gm.seq_embed(table, ok, float("nan"))
    assert e.value.code == -1
    with pytest.raises(GMetaError):
        gm.configure("wait", 2)
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=1 << 20)
    with pytest.raises(GMetaError) as e:
        small.seq_embed_grad(torch.ones(200_000, 8, device="cuda"), torch.zeros(200_000, dtype=torch.int32, device="cuda"), 50)
    assert e.value.code == -4 and "needs" in str(e.value)
    small.close()


@pytest.mark.gpu
def test_other_streams_than_the_contexts(gm):
    """Inputs made on another stream, results used there: both in order with the context's stream."""
    side = torch.cuda.Stream()
    table, tokens = torch.randn(1000, 64, device="cuda"), torch.randint(0, 1000, (50_000,), device="cuda").to(torch.int32)
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    own = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20, stream=torch.cuda.Stream().cuda_stream)
    for ctx in (gm, own):
        ctx.configure("wait", 0)
        with torch.cuda.stream(side):
            for _ in range(4):
                big = big @ big * 1e-4
            scaled = table * 2.0 + big[0, 0] * 0.0      # ready long after the call is made
            got = ctx.seq_embed(scaled, tokens) + 1.0
        side.synchronize()
        ctx.wait()
        ctx.configure("wait", 1)
        assert torch.equal(got, torch.nan_to_num(scaled)[tokens.long()] + 1.0)
    own.close()


@pytest.mark.gpu
def test_captured_calls_replay(gm):
    """Enqueued-only calls in a graph, replayed with other work between, each time against the eager result."""
    s = torch.cuda.Stream()
    ctx = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20, stream=s.cuda_stream)
    ctx.configure("wait", 0)
    rows, n, D = 3000, 20_000, 64
    tokens = torch.zeros(n, dtype=torch.int32, device="cuda")
    table, grad = torch.randn(rows, D, device="cuda"), torch.randn(n, D, device="cuda")
    out = torch.empty(n, D, device="cuda")
    lst = dict(emb_rows=torch.zeros(rows, dtype=torch.int64, device="cuda"), emb_grad=torch.zeros(rows, D, device="cuda"),
               n_emb_rows=torch.zeros(1, dtype=torch.int64, device="cuda"), capacity=rows)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        ctx.seq_embed(table, tokens, 2.0, out=out)
        ctx.seq_embed_grad(grad, tokens, rows, 1.0, out=lst)
    for i in range(4):
        tokens.copy_(torch.randint(0, rows, (n,)).to(torch.int32))
        grad.normal_()
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, table[tokens.long()] * 2.0)
        want = gm.seq_embed_grad(grad, tokens, rows, 1.0)
        k = int(want["n_emb_rows"])
        assert int(lst["n_emb_rows"]) == k and torch.equal(lst["emb_rows"][:k], want["emb_rows"][:k]) and torch.equal(lst["emb_grad"][:k], want["emb_grad"][:k])
    ctx.wait()
    del g
    ctx.close()


def test_workspace_of_the_largest_call_holds_every_smaller_one():
    from paper_2401_04338_amd import load_library
    size = load_library().gm_seq_embed_grad_bytes
    near = [2 ** e + d for e in (6, 13, 16, 19, 20, 21, 22, 24, 27) for d in (-4097, -1, 0, 1, 4097) if 2 ** e + d > 0]
    for dim in (1, 16, 128, 600):
        sizes = [size(n, dim) for n in sorted(near + [1_000_000, 600_000, 2 ** 31 - 1])]
        assert sizes == sorted(sizes) and sizes[0] > 0, dim


@pytest.mark.gpu
def test_a_context_for_many_tokens_takes_fewer(gm):
    """Workspace as the query says for a million tokens, and no more than a page beyond it: the calls on both sides of where the chunks of the sum change."""
    D, rows = 128, 5000
    small = type(gm)(1, [10], 4, 0, [4, 1], workspace_bytes=gm.lib.gm_seq_embed_grad_bytes(1_000_000, D) + 4096)
    for n in (1_000_000, 524_289, 524_288, 300_000, 8192, 1):
        tokens = torch.arange(n, device="cuda", dtype=torch.int32) % rows
        grad = torch.ones(n, D, device="cuda", dtype=torch.bfloat16)
        out = small.seq_embed_grad(grad, tokens, rows)
        k = int(out["n_emb_rows"])
        assert k == min(n, rows)
        assert torch.equal(out["emb_grad"][:k], torch.bincount(tokens.long(), minlength=k).float()[:k, None].expand(k, D))
    small.close()


@pytest.fixture(scope="module")
def large():
    from paper_2401_04338_amd import GMeta
    g = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=512 << 20)
    yield g
    g.close()


@pytest.mark.gpu
@pytest.mark.parametrize("n", [2 ** 20 - 1, 2 ** 20, 2 ** 21, 2 ** 21 + 1, 8_400_000])
@pytest.mark.parametrize("rows", [255, 70_000, 1 << 24])
def test_long_lists_where_the_sort_changes(large, n, rows):
    """From 2^20 tokens on the sort's tiles are twice as large, above 2^21 its passes narrower, above 2,048 tiles its table is scanned as a whole: whole numbers, exact."""
    gen = torch.Generator().manual_seed(n + rows)
    tokens = _tokens("skewed", n, rows, gen).cuda()
    keep = tokens >= 0
    counts = torch.bincount(tokens[keep].long().cpu(), minlength=rows).cuda()
    want = counts.nonzero()[:, 0]
    place = (torch.arange(n, device="cuda") * 31 % 509).float()                       # (sums below 2^24 where a row has 32,000 tokens or fewer)
    sums = torch.zeros(rows, dtype=torch.float64).index_add_(0, tokens[keep].long().cpu(), place[keep].double().cpu()).cuda()
    for grad, total in ((torch.ones(n, 1, device="cuda"), counts.double()), (place[:, None], sums)):
        out = large.seq_embed_grad(grad, tokens, rows)
        k = int(out["n_emb_rows"])
        assert k == len(want) and torch.equal(out["emb_rows"][:k], want)
        exact = total[want] < 2 ** 24
        assert exact.sum() > 100 and torch.equal(out["emb_grad"][:k, 0].double()[exact], total[want][exact])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
@pytest.mark.parametrize("dim", [3, 36, 128])
@pytest.mark.parametrize("n", [400_000, 700_000])
def test_hot_rows_of_long_lists(large, n, dim, dtype):
    """Rows that fill whole workgroups of the sum, and rows of one token, in chunks of 16 and of 64: small whole numbers, whose sums are exact in any order."""
    gen, rows = torch.Generator().manual_seed(n + dim), 90_000
    tokens = torch.randint(0, rows, (n,), generator=gen)
    at = torch.rand(n, generator=gen)
    for row, share in ((17, 0.3), (rows - 1, 0.45), (0, 0.5), (40_000, 0.502)):
        tokens[(at < share) & (at >= {17: 0.0, rows - 1: 0.3, 0: 0.45, 40_000: 0.5}[row])] = row
    tokens[at > 0.95] = -1
    grad = torch.randint(-8, 9, (n, dim), generator=gen).to(dtype)
    grad[tokens < 0] = float("nan")
    tokens, grad = tokens.to(torch.int32).cuda(), grad.cuda()
    keep = tokens >= 0
    sums = torch.zeros(rows, dim, dtype=torch.float64).index_add_(0, tokens[keep].long().cpu(), grad[keep].double().cpu()).cuda()
    want = torch.unique(tokens[keep].long())
    out = large.seq_embed_grad(grad, tokens, rows, 0.5)
    k = int(out["n_emb_rows"])
    assert k == len(want) and torch.equal(out["emb_rows"][:k], want) and torch.equal(out["emb_grad"][:k].double(), sums[want] * 0.5)
    table = torch.randint(-100, 100, (rows, dim), device="cuda").float()
    full = table.double() + sums * 0.5
    assert torch.equal(large.seq_embed_grad(grad, tokens, rows, 0.5, table=table).double(), full)


@pytest.mark.gpu
def test_a_list_of_other_rows_is_refused(gm):
    """A list of an earlier call with wider rows holds enough values, but not in rows of this call's width."""
    tokens = torch.arange(10, dtype=torch.int32, device="cuda")
    out = gm.seq_embed_grad(torch.ones(10, 16, device="cuda"), tokens, 50)
    assert out["emb_grad"].shape == (10, 16)
    with pytest.raises(ValueError):
        gm.seq_embed_grad(torch.ones(10, 8, device="cuda"), tokens, 50, out=out)
    with pytest.raises(ValueError):
        gm.seq_embed_grad(torch.ones(11, 16, device="cuda"), torch.arange(11, dtype=torch.int32, device="cuda"), 50, out=dict(out, capacity=11))
    flat = dict(out, emb_grad=torch.zeros(80, device="cuda"))
    assert (gm.seq_embed_grad(torch.ones(10, 8, device="cuda"), tokens, 50, out=flat)["emb_grad"] == 1).all()
    again = gm.seq_embed_grad(2 * torch.ones(10, 16, device="cuda"), tokens, 50, out=out)
    assert again is out and (out["emb_grad"] == 2).all()
