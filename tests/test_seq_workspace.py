"""What the calls on histories write lies in the workspace that the library names a size for: their launches looked at without a GPU (seq_workspace.cpp), and calls in contexts of just
that size."""
import os
import subprocess

import pytest
import torch

from tests import block_ref as B
from tests import seq_ref as R

gpu = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """seq_workspace.cpp, built against the library."""
    from paper_2401_04338_amd import LIB_PATH, build
    if not os.path.exists(LIB_PATH):
        build.build(verbose=False)
    where, out = os.path.dirname(LIB_PATH), str(tmp_path_factory.mktemp("launches") / "seq_workspace")
    subprocess.run([os.environ.get("HIPCC", "/opt/rocm/bin/hipcc"), "-std=c++17", "-O1", "-x", "hip", "--offload-host-only", "-rdynamic", os.path.join(HERE, "seq_workspace.cpp"), "-o", out,
                    f"-L{where}", "-lgmeta", f"-Wl,-rpath,{where}", "-ldl"], check=True)
    return out


@pytest.mark.parametrize("call", ["norm", "glu", "attend"])
def test_launches_stay_inside(launches, call):
    r = subprocess.run([launches, call], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True, timeout=300)
    assert r.returncode == 0, r.stdout


@gpu
@pytest.mark.parametrize("n,Ch,dtype", [(2000, 512, torch.float32), (4100, 250, torch.bfloat16), (1024, 1024, torch.bfloat16), (1024, 1025, torch.bfloat16), (1000, 2048, torch.bfloat16),
                                        (3000, 1030, torch.bfloat16), (700, 4096, torch.bfloat16), (1024, 8192, torch.bfloat16), (300, 8200, torch.bfloat16), (1024, 2048, torch.float32),
                                        (1500, 2049, torch.float32), (1024, 4096, torch.float32), (900, 4097, torch.float32)])
def test_norm_gradient_in_the_size_it_names(n, Ch, dtype):
    """Rows of every form, a workgroup a row among them, whose weights' gradients are summed over as many workgroups as there are rows."""
    from paper_2401_04338_amd import GMeta
    from paper_2401_04338_amd.binding import load_library
    need = load_library().gm_seq_norm_grad_bytes(n, Ch)
    exact, roomy = (GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=size) for size in (need + 4096, 256 << 20))
    gen = torch.Generator().manual_seed(Ch)
    x, dy, w = torch.randn(n, Ch, generator=gen).to(dtype), (torch.randn(n, Ch, generator=gen) * 0.1).to(dtype), torch.randn(Ch, generator=gen)
    xc, dyc, wc = x.cuda(), dy.cuda(), w.cuda()
    stats = exact.seq_norm(xc)[2]
    got, want = (g.seq_norm_grad(dyc, xc, stats, wc) for g in (exact, roomy))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ref = B.norm_grad(dy, x, stats.cpu(), w, None)
    for i, name in enumerate(("ds", "dweight", "dbias")):
        R.within(got[i], ref[i], ref[i + 3], name)
    for g in (exact, roomy):
        g.close()


@gpu
@pytest.mark.parametrize("n,K,N,dtype", [(817, 64, 1024, torch.float32), (127, 512, 2048, torch.bfloat16), (400, 64, 4096, torch.bfloat16), (90, 8, 16_384, torch.bfloat16),
                                         (2048, 64, 1024, torch.float32)])
def test_feed_forward_gradient_in_the_size_it_names(n, K, N, dtype):
    """Wide rows and few of them, with biases: a row of sums for every workgroup holds all of d_out."""
    from paper_2401_04338_amd import GMeta
    roomy = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=256 << 20)
    exact = GMeta(1, [10], 4, 0, [4, 1], workspace_bytes=roomy.lib.gm_seq_glu_grad_bytes(roomy._ctx, n, K, N, int(dtype == torch.bfloat16)) + 4096)
    gen = torch.Generator().manual_seed(N)
    x, wg, wu, gate, up, dy = (torch.randn(*s, generator=gen).to(dtype).cuda() for s in ((n, K), (K, N), (K, N), (n, N), (n, N), (n, N)))
    got, want = (g.seq_glu_grad(dy, x, wg, wu, gate, up, "silu", bias=True) for g in (exact, roomy))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    ref = B.glu_grad(dy, x, wg, wu, gate, up, "silu")
    for i, name in enumerate(("dx", "dw_gate", "dw_up", "db_gate", "db_up")):
        R.within(got[i], ref[i].cpu(), ref[i + 5].cpu(), name)
    for g in (exact, roomy):
        g.close()
