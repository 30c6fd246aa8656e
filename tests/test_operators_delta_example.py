"""The example that trains a block with matrix states with AdamW and serves it (examples/delta_block.py)."""
import os
import sys

import numpy as np
import pytest

import operator_reference as ref

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def block64(block, params, x, residual, lengths):
    """The block in 64 bits, for torch's own differentiation on the CPU."""
    import torch
    import torch.nn.functional as F
    s = x + residual
    n = s * (s.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * params["norm"]
    q, k, v, a, b = (n @ params["projection"].T).split(block.split, -1)

    def unit(t):  # heads of length 1, as often as value heads share them
        t = t.unflatten(-1, (block.key_heads, block.dk))
        t = t * (t.pow(2).mean(-1, keepdim=True) + 1e-6).rsqrt() * block.dk ** -0.5
        return t.repeat_interleave(block.heads // block.key_heads, -2)
    q, k, v = unit(q), unit(k), v.unflatten(-1, (block.heads, block.dv))
    g, beta = -params["rate"].exp() * F.softplus(a), torch.sigmoid(b)
    S, out = torch.zeros(x.shape[1], block.heads, block.dk, block.dv, dtype=x.dtype), []
    for t in range(x.shape[0]):
        W = S * g[t].exp()[..., None, None]
        u = beta[t][..., None] * (v[t] - torch.einsum("bhkv,bhk->bhv", W, k[t]))
        new = W + torch.einsum("bhk,bhv->bhkv", k[t], u)
        live = (t < lengths)[:, None, None]
        out.append(torch.where(live, torch.einsum("bhkv,bhk->bhv", new, q[t]) * block.dk ** -0.5, torch.zeros_like(v[t])))
        S = torch.where(live[..., None], new, S)
    return torch.stack(out).flatten(2) @ params["output"].T, s


def test_gradients_and_update_of_the_whole_block(cuda_device):
    """In fp32 the gradients are within 2e-4 (of each tensor's largest) of those in 64 bits: sums of at most 70 x 3 x 96
    products, each off by a few units of 2^-24 and the delta rule's by 2^-18 at most, through eight operators.  One
    AdamW step with these gradients then is the formula's."""
    import torch
    from delta_block import Block, Trainer
    T, B, D = 70, 3, 96
    block = Block(D, 4, 32, 24, torch.float32, seed=5)
    x, residual, dy, ds = (torch.randn(T, B, D, device="cuda") for _ in range(4))
    lengths = torch.tensor([70, 17, 0], device="cuda", dtype=torch.int32)
    y, kept = block.forward(x, residual, lengths)
    dx, grads = block.backward(dy, kept, ds)
    p64 = {k: v.double().cpu().requires_grad_() for k, v in block.parameters().items()}
    x64, r64 = x.double().cpu().requires_grad_(), residual.double().cpu()
    y64, s64 = block64(block, p64, x64, r64, lengths.cpu())
    (y64 * dy.double().cpu()).sum().add((s64 * ds.double().cpu()).sum()).backward()
    for name, got, want in [("y", y, y64.detach()), ("dx", dx, x64.grad)] + [(k, grads[k], p64[k].grad) for k in grads]:
        assert float((got.double().cpu() - want).abs().max()) <= 2e-4 * float(want.abs().max()), name
    before = {k: ref.f64(v) for k, v in block.parameters().items()}
    trainer = Trainer(block, 32, lr=1e-2, weight_decay=0.1)
    trainer.update(grads)
    for k, v in block.parameters().items():
        g = ref.f64(grads[k])  # the first step: m / (1 - b1) = g, v / (1 - b2) = g^2
        want = before[k] * (1 - 1e-3) - 1e-2 * g / (np.abs(g) + 1e-8)
        assert np.abs(ref.f64(v) - want).max() <= 40 * ref.U32 * (np.abs(before[k]).max() + 1e-2), k
        if k in block.copies:
            assert torch.equal(block.copies[k], v.to(block.copies[k].dtype))


def test_serving_goes_on_where_the_sequence_ends(cuda_device):
    """Ticks with idle slots in between give the outputs and states of the sequence, in fp32 to 1e-4 of the largest."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, rms_norm
    from delta_block import Block, Server
    T, B, D = 70, 5, 64
    block = Block(D, 2, 32, 32, torch.float32, seed=6)
    server = Server(block, 8)
    server.state.normal_()  # what an earlier stream left
    x, residual = (torch.randn(T, B, D, device="cuda") for _ in range(2))
    slots = torch.tensor([7, 0, 3, 4, 1], device="cuda", dtype=torch.int32)
    idle = server.state[[2, 5, 6]].clone()
    got = torch.stack([server.tick(x[t], residual[t].clone(), slots, torch.full((B,), t == 0, device="cuda"))
                       for t in range(T)])
    want, kept = block.forward(x, residual)
    q1, k1, v, g, beta = kept[7:12]
    last = delta_scan(q1, k1, v, g, beta)[1]
    assert float((got - want).abs().max()) <= 1e-4 * float(want.abs().max())
    assert float((server.state[slots.long()] - last).abs().max()) <= 1e-4 * float(last.abs().max())
    assert torch.equal(server.state[[2, 5, 6]], idle)


@pytest.mark.parametrize("bits", [8, 32])
def test_example_runs(cuda_device, bits):
    """Losses are finite; served outputs are those of the sequences but for roundings to 16 bits of q, k, v, o and y on
    either way (2^-8 each at most, 5 of them, and their products)."""
    from delta_block import main
    losses, far = main(width=256, heads=4, streams=4, steps=70, updates=4, bits=bits)
    assert np.isfinite(losses).all() and far < 10 * 2.0 ** -8
