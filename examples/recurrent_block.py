"""A gated-linear-recurrence block, trained on sequences and served token by
token with the operators of paper_1905_00689_gb300.

    x' = x + residual;  z = rms_norm(x') P^T;  h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigma(i_t) v_t

v, r and i are the thirds of z, a_t follows from r and the channel's decay.

Training runs over whole sequences [T, B, D] of their own lengths; the block's
gradients are written out, and the scan's go straight into the slices of the
projection's.  Serving keeps P in 4 bits and a pool of streams' states: each
tick is three launches for the streams that have a token.

    python examples/recurrent_block.py [--width 512 --streams 16 --steps 64 --updates 20]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1905_00689_gb300 import (gated_scan, gated_scan_backward, gated_scan_states, gated_step, rms_norm,
                                    rms_norm_backward, rms_norm_quant, w4_matvec, w4_quantize)

EPS = 1e-6


class Block:
    """The parameters in fp32; products and sequences in `dtype`."""

    def __init__(self, width, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.width, self.dtype = width, dtype
        self.norm = torch.ones(width, device=device)
        self.projection = torch.randn(3 * width, width, generator=g, device=device) * width ** -0.5
        self.decay = torch.rand(width, generator=g, device=device) - 5.0

    def parameters(self):
        return {"norm": self.norm, "projection": self.projection, "decay": self.decay}

    def forward(self, x, residual, lengths=None):
        """y [T, B, D] and what backward() needs."""
        T, B, D = x.shape
        rstd = torch.empty(T, B, device=x.device)
        n, total = rms_norm(x, self.norm, residual, eps=EPS, rstd=rstd)
        z = n @ self.projection.to(self.dtype).T
        states = gated_scan_states(T, B, D, x.device)
        y, _ = gated_scan(z[..., :D], z[..., D:2 * D], z[..., 2 * D:], self.decay, lengths=lengths, states=states)
        return y, (n, total, rstd, z, states, lengths)

    def backward(self, dy, kept, dtotal=None):
        """Gradients of x (and of the residual alike) and of the parameters."""
        n, total, rstd, z, states, lengths = kept
        D = self.width
        dz = torch.empty_like(z)
        _, _, _, ddecay, _ = gated_scan_backward(
            dy, z[..., :D], z[..., D:2 * D], z[..., 2 * D:], self.decay, states, lengths=lengths,
            dx=dz[..., :D], dr=dz[..., D:2 * D], di=dz[..., 2 * D:])
        dn = dz @ self.projection.to(self.dtype)
        dprojection = (dz.flatten(0, 1).T @ n.flatten(0, 1)).float()
        dx, dnorm = rms_norm_backward(dn, total, self.norm, rstd, dtotal)
        return dx, {"norm": dnorm, "projection": dprojection, "decay": ddecay}


class Server:
    """The block for single tokens of many streams: P in 4 bits, a state per slot."""

    def __init__(self, block, slots, group=128):
        self.block = block
        self.weight = w4_quantize(block.projection, group=group)
        self.state = torch.zeros(slots, block.width, device=block.norm.device)

    def tick(self, x, residual, slots, fresh=None):
        """One token for each of the streams in `slots`; `fresh` marks those that begin.  residual becomes x + residual."""
        D = self.block.width
        q, scales, _ = rms_norm_quant(x, self.block.norm, residual, eps=EPS, residual_out=residual)
        z = w4_matvec(q, self.weight, x_scale=scales, out_dtype=self.block.dtype)
        return gated_step(z[:, :D], z[:, D:2 * D], z[:, 2 * D:], self.block.decay, self.state, slots=slots, reset=fresh)


def main(width=512, streams=16, steps=64, updates=20, rate=0.02, dtype=torch.bfloat16):
    block = Block(width, dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, residual = (torch.randn(steps, streams, width, generator=g, device="cuda").to(dtype) for _ in range(2))
    lengths = torch.randint(1, steps + 1, (streams,), generator=g, device="cuda", dtype=torch.int32)
    lengths[0] = steps
    # what the block learns: the outputs of another one
    target = Block(width, dtype, seed=2).forward(x, residual, lengths)[0].float()
    count = float(lengths.sum()) * width
    losses = []
    for _ in range(updates):
        y, kept = block.forward(x, residual, lengths)
        error = y.float() - target  # (zero past a stream's length on both sides)
        losses.append(float((error ** 2).sum() / count))
        _, grads = block.backward((error * (2.0 / count)).to(dtype), kept)
        for name, p in block.parameters().items():
            p -= rate * p.norm() / (grads[name].norm() + 1e-20) * grads[name]  # a step of that share of p's length

    want, _ = block.forward(x, residual)
    server = Server(block, 2 * streams)
    slots = torch.randperm(2 * streams, generator=g, device="cuda")[:streams].to(torch.int32)
    got = torch.empty_like(want)
    for t in range(steps):
        fresh = torch.full((streams,), t == 0, device="cuda")
        got[t] = server.tick(x[t], residual[t].clone(), slots, fresh)
    far = float((got.float() - want.float()).norm() / want.float().norm())
    return losses, far


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 512), ("streams", 16), ("steps", 64), ("updates", 20)):
        p.add_argument(f"--{name}", type=int, default=value)
    losses, far = main(**vars(p.parse_args()))
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f} after {len(losses)} updates; "
          f"served with a 4-bit projection: outputs {100 * far:.1f}% away (norm) from those of the trained block")
