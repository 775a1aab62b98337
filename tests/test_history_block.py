"""The calls of a self-attention block run together, as examples/history_block.py has them: against the block in 64 bits with the library's derivatives, and served in pieces."""
import math
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
U = 2.0 ** -24


def _plain(w, x, lens, H, G, D, hidden):
    """The block in 64 bits, history by history, by torch's own operators on the CPU."""
    F = torch.nn.functional
    width, outs, at = H * D, [], 0
    for n in lens:
        rows = x[at:at + n]
        at += n
        if not n:
            continue
        n1 = F.layer_norm(rows, (width,), w["norm1"], w["bias1"])
        q, k, v = (n1 @ w["qkv"]).view(n, H + 2 * G, D).split([H, G, G], 1)
        k, v = k.repeat_interleave(H // G, 1), v.repeat_interleave(H // G, 1)
        s = torch.matmul(q.permute(1, 0, 2), k.permute(1, 2, 0)) / D ** 0.5
        s = s.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -math.inf)
        o = torch.matmul(torch.softmax(s, 2), v.permute(1, 0, 2)).permute(1, 0, 2).reshape(n, width)
        s = rows + o @ w["out"]
        n2 = F.layer_norm(s, (width,), w["norm2"], w["bias2"])
        y = F.silu(n2 @ w["gate_up"][:, :hidden] + w["b_gate"]) * (n2 @ w["gate_up"][:, hidden:] + w["b_up"])
        outs.append(s + y @ w["down"])
    return torch.cat(outs)


@pytest.mark.gpu
def test_forward_and_every_gradient():
    """fp32.  A value goes through seven products and sums of up to 256 terms and two norms: some 2,000 roundings of 2^-24 of the magnitudes that take part, 1e-4 of the largest
    entry of the array at the very most; gradients likewise, with sums over all rows."""
    import history_block as B
    from paper_2401_04338_amd import GMeta
    gm = GMeta(1, [16], 4, 0, [4, 1], workspace_bytes=64 << 20)
    block = B.HistoryBlock(gm, torch.Generator(device="cuda").manual_seed(3), torch.float32)
    lens = [37, 0, 1, 130, 5]
    gen = torch.Generator().manual_seed(1)
    x, dout = torch.randn(sum(lens), B.WIDTH, generator=gen), torch.randn(sum(lens), B.WIDTH, generator=gen)
    out, kept = block.forward(x.cuda(), B.packed(lens), max(lens))
    dx, g = block.backward(dout.cuda(), kept)
    w = {k: v.detach().cpu().double().requires_grad_() for k, v in block.w.items()}
    xr = x.double().requires_grad_()
    ref = _plain(w, xr, lens, B.HEADS, B.KV_HEADS, B.HEAD_DIM, B.HIDDEN)
    grads = torch.autograd.grad((ref * dout.double()).sum(), [xr, *w.values()])
    for name, got, want in (("out", out, ref), ("x", dx, grads[0]), *((k, g[k], t) for k, t in zip(w, grads[1:]))):
        off = float((got.detach().cpu().double() - want.detach()).abs().max() / want.detach().abs().max())
        assert off < 2000 * U, (name, off)
    gm.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=["fp32", "bf16"])
def test_what_is_served_in_pieces_is_what_was_trained(dtype):
    import history_block as B
    losses, off = B.run(steps=3, users=40, dtype=dtype, say=lambda *a: None)
    assert all(math.isfinite(v) for v in losses)
    # The same rows through the same products; the attention takes its sums in other orders, and in bf16 that moves roundings (2^-8 each) of six arrays on the way
    assert off < (2000 * U if dtype == torch.float32 else 6 * 2.0 ** -8)
