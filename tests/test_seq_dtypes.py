"""What the kernels write as fp32 is made as fp32, whatever type torch makes by default."""
import pytest
import torch

gpu = pytest.mark.gpu
DEFAULTS = pytest.mark.parametrize("default", [torch.bfloat16, torch.float16, torch.float64], ids=["bf16", "fp16", "fp64"])


@pytest.fixture
def default_type(default):
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    yield default
    torch.set_default_dtype(before)


def _calls(gm, device, dtype=torch.bfloat16):
    """Every call that makes arrays of fp32 by itself: its name, and those arrays."""
    f32 = dict(dtype=torch.float32, device=device)
    gen = torch.Generator(device=device).manual_seed(3)
    r = lambda *s: torch.randn(*s, generator=gen, **f32).to(dtype)  # noqa: E731
    n, Ch, K, N = 70, 40, 16, 24
    x, dy, weight = r(n, Ch), r(n, Ch), torch.ones(Ch, **f32)
    off = torch.tensor([0, 30, 30, n], device=device)
    y, s, stats = gm.seq_norm(x, weight, weight, residual=dy)
    yield "norm", (stats,)
    yield "norm_grad", gm.seq_norm_grad(dy, s, stats, weight)[1:]
    x2, w, d = r(n, K), r(K, 2 * N), r(n, N)
    bias = torch.zeros(N, **f32)
    _, gate, up = gm.seq_glu(x2, w[:, :N], w[:, N:], b_gate=bias, b_up=bias, keep=True)
    yield "glu_grad", gm.seq_glu_grad(d, x2, w[:, :N], w[:, N:], gate, up, bias=True)[3:]
    h, last = gm.seq_scan(x, dy, off, 40)
    h0 = torch.zeros(3, Ch, **f32)
    yield "scan", (last,)
    yield "scan_grad", (gm.seq_scan_grad(dy, x, dy, h, off, 40, h0=h0, dlast=torch.zeros_like(h0))[2],)
    q, k = r(n, 2, 16), r(n, 1, 16)
    for causal in (False, True):
        yield "attend", (gm.seq_attend(q, k, k, off, off, 40, 40, causal=causal)[1],)
    tokens = torch.arange(n, dtype=torch.int32, device=device) % 9
    yield "embed_grad", (gm.seq_embed_grad(dy, tokens, 10)["emb_grad"],)


@DEFAULTS
def test_arrays_are_made_as_fp32(default_type, monkeypatch):
    """Without a GPU: nothing is called, the arrays that would be written are looked at."""
    from paper_2401_04338_amd import GMeta, binding
    monkeypatch.setattr(binding, "_checked", lambda t, dtype, name, device=None: t)
    gm = GMeta.__new__(GMeta)
    gm.lib, gm.device, gm._seq_call = binding.load_library(), torch.device("cpu"), lambda *args: None
    for name, made in _calls(gm, gm.device):
        assert all(t.dtype is torch.float32 for t in made), name


@gpu
@DEFAULTS
def test_results_do_not_depend_on_the_default(default_type):
    from paper_2401_04338_amd import GMeta
    gm = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=64 << 20)
    device = torch.device("cuda", 0)
    got = list(_calls(gm, device))
    torch.set_default_dtype(torch.float32)
    for (name, made), (_, want) in zip(got, _calls(gm, device)):
        n = 9 if name == "embed_grad" else None     # (rows of the list that are written)
        assert all(a.dtype is torch.float32 and torch.equal(a[:n], b[:n]) for a, b in zip(made, want)), name
    gm.close()
