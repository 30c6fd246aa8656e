"""The example that trains and serves a block with the operators (examples/recurrent_block.py)."""
import os
import sys

import pytest

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def block64(params, x, residual, lengths):
    """The block in 64 bits, for torch's own differentiation on the CPU."""
    import torch
    import torch.nn.functional as F
    D = x.shape[-1]
    s = x + residual
    n = s * (s.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * params["norm"]
    v, r, i = (n @ params["projection"].T).split(D, -1)
    h, out = torch.zeros_like(x[0]), []
    for t in range(x.shape[0]):
        log_a = -8.0 * F.softplus(params["decay"]) * torch.sigmoid(r[t])
        new = log_a.exp() * h + (-torch.expm1(2 * log_a)).sqrt() * torch.sigmoid(i[t]) * v[t]
        live = (t < lengths)[:, None]
        h = torch.where(live, new, h)
        out.append(torch.where(live, new, torch.zeros_like(new)))
    return torch.stack(out), s


def test_gradients_of_the_whole_block(cuda_device):
    """In fp32 the gradients are within 1e-4 (of each tensor's largest) of those in 64 bits: sums of at most 40 x 3
    x 64 products, each off by a few units of 2^-24, through five operators."""
    import torch
    from recurrent_block import Block
    T, B, D = 40, 3, 64
    block = Block(D, torch.float32, seed=5)
    x, residual, dy, ds = (torch.randn(T, B, D, device="cuda") for _ in range(4))
    lengths = torch.tensor([40, 17, 0], device="cuda", dtype=torch.int32)
    y, kept = block.forward(x, residual, lengths)
    dx, grads = block.backward(dy, kept, ds)
    p64 = {k: v.double().cpu().requires_grad_() for k, v in block.parameters().items()}
    x64, r64 = x.double().cpu().requires_grad_(), residual.double().cpu()
    y64, s64 = block64(p64, x64, r64, lengths.cpu())
    (y64 * dy.double().cpu()).sum().add((s64 * ds.double().cpu()).sum()).backward()
    for name, got, want in [("y", y, y64.detach()), ("dx", dx, x64.grad)] + [(k, grads[k], p64[k].grad) for k in grads]:
        assert float((got.double().cpu() - want).abs().max()) <= 1e-4 * float(want.abs().max()), name


def test_serving_goes_on_where_the_sequence_ends(cuda_device):
    """Ticks with idle slots in between give the states of one scan over the same 8-bit norm outputs and 4-bit matrix:
    the same arithmetic in fp32, 1e-4 of the largest."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, rms_norm_quant, w4_matvec
    from recurrent_block import Block, Server
    T, B, D = 9, 5, 96
    block = Block(D, torch.float32, seed=6)
    server = Server(block, 8, group=32)
    server.state.normal_()  # what an earlier stream left
    x, residual = (torch.randn(T, B, D, device="cuda") for _ in range(2))
    slots = torch.tensor([7, 0, 3, 4, 1], device="cuda", dtype=torch.int32)
    idle = server.state[[2, 5, 6]].clone()
    got = torch.stack([server.tick(x[t], residual[t].clone(), slots, torch.full((B,), t == 0, device="cuda"))
                       for t in range(T)])
    q, scales, _ = rms_norm_quant(x.flatten(0, 1), block.norm, residual.flatten(0, 1), eps=1e-6)
    z = w4_matvec(q, server.weight, x_scale=scales, out_dtype=torch.float32).view(T, B, 3 * D)
    want, last = gated_scan(z[..., :D], z[..., D:2 * D], z[..., 2 * D:], block.decay)
    assert float((got - want).abs().max()) <= 1e-4 * float(want.abs().max())
    assert float((server.state[slots.long()] - last).abs().max()) <= 1e-4 * float(last.abs().max())
    assert torch.equal(server.state[[2, 5, 6]], idle)


def test_example_learns_and_serves(cuda_device):
    """The loss falls, and the served outputs stay within the roundings of P to 4 bits (a step is 1/15 of a group's
    range: about 10% of a value's size, norm by norm) and of the norm's output to 8 bits (3%)."""
    from recurrent_block import main
    losses, far = main(width=256, streams=8, steps=33, updates=12)
    assert losses[-1] < 0.9 * losses[0]
    assert far < 0.25
