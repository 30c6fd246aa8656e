"""A block whose state is a matrix for each head (the gated delta rule), trained with AdamW on sequences and served token by
token with the operators of paper_1905_00689_gb300.

    x' = x + residual;  z = rms_norm(x') P^T = (q, k, v, a, b)
    g = -e^rate softplus(a);  beta = sigmoid(b);  q and k of length 1
    o = delta rule of (q, k, v, g, beta);  y = o W^T

Training runs over whole sequences [T, B, width] of their own lengths; the block's gradients are written out.  The
parameters are kept in 32 bits; the update writes their 16-bit copies, which the next pass computes with.  Serving keeps
a pool of streams' states: a tick takes one token of some of them.

    python examples/delta_block.py [--width 512 --heads 4 --streams 8 --steps 96 --updates 20 --bits 8]
"""
import argparse
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1905_00689_gb300 import (AdamWState, adamw_step, delta_scan, delta_scan_backward, delta_scan_states, delta_step,
                                    rms_norm, rms_norm_backward)

EPS = 1e-6


class Block:
    """The parameters in fp32, sequences and products in `dtype`; `heads` value heads, two to a query and key head."""

    def __init__(self, width, heads, dk=64, dv=64, dtype=torch.bfloat16, seed=0, device="cuda"):
        g = torch.Generator(device=device).manual_seed(seed)
        self.width, self.heads, self.key_heads, self.dk, self.dv, self.dtype = width, heads, heads // 2, dk, dv, dtype
        self.split = (self.key_heads * dk, self.key_heads * dk, heads * dv, heads, heads)
        self.norm = torch.ones(width, device=device)
        self.projection = torch.randn(sum(self.split), width, generator=g, device=device) * width ** -0.5
        self.output = torch.randn(width, heads * dv, generator=g, device=device) * (heads * dv) ** -0.5
        self.rate = torch.rand(heads, generator=g, device=device) - 3.0
        self.unit = torch.full((dk,), dk ** -0.5, device=device)  # a norm's weight for rows of length 1
        self.copies = {"projection": self.projection.to(dtype), "output": self.output.to(dtype)}

    def parameters(self):
        return {"norm": self.norm, "projection": self.projection, "output": self.output, "rate": self.rate}

    def inputs(self, z):
        """What the delta rule takes of z [..., sum(split)]: q and k before their norms, v, g, beta, a."""
        q, k, v, a, b = z.split(self.split, -1)
        q, k = (t.unflatten(-1, (self.key_heads, self.dk)).contiguous() for t in (q, k))
        a, beta = a.float(), torch.sigmoid(b.float())
        return q, k, v.unflatten(-1, (self.heads, self.dv)), -self.rate.exp() * torch.nn.functional.softplus(a), beta, a

    def forward(self, x, residual, lengths=None):
        """y [T, B, width] and what backward() needs."""
        rstd, q_rstd, k_rstd = (torch.empty(*x.shape[:2], *n, device=x.device) for n in ((), (self.key_heads,), (self.key_heads,)))
        n, total = rms_norm(x, self.norm, residual, eps=EPS, rstd=rstd)
        z = n @ self.copies["projection"].T
        q, k, v, g, beta, a = self.inputs(z)
        q1, _ = rms_norm(q, self.unit, eps=EPS, rstd=q_rstd)
        k1, _ = rms_norm(k, self.unit, eps=EPS, rstd=k_rstd)
        states = delta_scan_states(q1, v)
        o, _ = delta_scan(q1, k1, v, g, beta, lengths=lengths, states=states)
        y = o.flatten(2) @ self.copies["output"].T
        return y, (n, total, rstd, q, k, q_rstd, k_rstd, q1, k1, v, g, beta, a, states, o, lengths)

    def backward(self, dy, kept, dtotal=None):
        """Gradients of x (and of the residual alike) and of the parameters."""
        n, total, rstd, q, k, q_rstd, k_rstd, q1, k1, v, g, beta, a, states, o, lengths = kept
        do = (dy @ self.copies["output"]).unflatten(-1, (self.heads, self.dv))
        doutput = (dy.flatten(0, 1).T @ o.flatten(0, 1).flatten(1)).float()
        dz = torch.empty(*dy.shape[:2], sum(self.split), dtype=dy.dtype, device=dy.device)
        into_q, into_k, into_v, into_a, into_b = dz.split(self.split, -1)
        dq1, dk1, _, dg, dbeta, _ = delta_scan_backward(do, q1, k1, v, g, beta, states, lengths=lengths,
                                                        dv=into_v.unflatten(-1, (self.heads, self.dv)))
        into_q.copy_(rms_norm_backward(dq1, q, self.unit, q_rstd)[0].flatten(2))
        into_k.copy_(rms_norm_backward(dk1, k, self.unit, k_rstd)[0].flatten(2))
        into_a.copy_(-self.rate.exp() * torch.sigmoid(a) * dg)
        into_b.copy_(dbeta * beta * (1 - beta))
        dprojection = (dz.flatten(0, 1).T @ n.flatten(0, 1)).float()
        dx, dnorm = rms_norm_backward(dz @ self.copies["projection"], total, self.norm, rstd, dtotal)
        return dx, {"norm": dnorm, "projection": dprojection, "output": doutput, "rate": (dg * g).sum((0, 1))}


class Trainer:
    """AdamW on a block's parameters, with averages in 32 or 8 bits; it writes the block's 16-bit copies."""

    def __init__(self, block, bits=32, **rates):
        self.block, self.rates, self.step = block, rates, 0
        self.names = list(block.parameters())
        self.state = AdamWState.zeros(block.parameters().values(), bits)

    def update(self, grads):
        self.step += 1
        params = self.block.parameters()
        adamw_step([params[n] for n in self.names], [grads[n] for n in self.names], self.state, self.step,
                   copies=[self.block.copies.get(n) for n in self.names], **self.rates)


class Server:
    """The block for single tokens of many streams: a matrix per slot and head."""

    def __init__(self, block, slots):
        self.block = block
        self.state = torch.zeros(slots, block.heads, block.dk, block.dv, device=block.norm.device)

    def tick(self, x, residual, slots, fresh=None):
        """One token for each of the streams in `slots`; `fresh` marks those that begin.  residual becomes x + residual."""
        n, _ = rms_norm(x, self.block.norm, residual, eps=EPS, residual_out=residual)
        q, k, v, g, beta, _ = self.block.inputs(n @ self.block.copies["projection"].T)
        q, _ = rms_norm(q, self.block.unit, eps=EPS)
        k, _ = rms_norm(k, self.block.unit, eps=EPS)
        o = delta_step(q, k, v, g, beta, self.state, slots=slots, reset=fresh)
        return o.flatten(1) @ self.block.copies["output"].T


def main(width=512, heads=4, streams=8, steps=96, updates=20, bits=8, dtype=torch.bfloat16):
    block = Block(width, heads, dtype=dtype)
    g = torch.Generator(device="cuda").manual_seed(1)
    x, residual = (torch.randn(steps, streams, width, generator=g, device="cuda").to(dtype) for _ in range(2))
    lengths = torch.randint(1, steps + 1, (streams,), generator=g, device="cuda", dtype=torch.int32)
    lengths[0] = steps
    # what the block learns: the outputs of another one
    target = Block(width, heads, dtype=dtype, seed=2).forward(x, residual, lengths)[0].float()
    count = float(lengths.sum()) * width
    trainer, losses = Trainer(block, bits, lr=1e-2, weight_decay=0.01), []
    for _ in range(updates):
        y, kept = block.forward(x, residual, lengths)
        error = y.float() - target  # (zero past a stream's length on both sides)
        losses.append(float((error ** 2).sum() / count))
        _, grads = block.backward((error * (2.0 / count)).to(dtype), kept)
        trainer.update(grads)

    want, _ = block.forward(x, residual)
    server = Server(block, 2 * streams)
    slots = torch.randperm(2 * streams, generator=g, device="cuda")[:streams].to(torch.int32)
    got = torch.empty_like(want)
    for t in range(steps):
        got[t] = server.tick(x[t], residual[t].clone(), slots, torch.full((streams,), t == 0, device="cuda"))
    return losses, float((got.float() - want.float()).norm() / want.float().norm())


if __name__ == "__main__":
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("width", 512), ("heads", 4), ("streams", 8), ("steps", 96), ("updates", 20), ("bits", 8)):
        p.add_argument(f"--{name}", type=int, default=value)
    losses, far = main(**vars(p.parse_args()))
    print(f"loss {losses[0]:.5f} -> {losses[-1]:.5f} after {len(losses)} updates; "
          f"served token by token: outputs {100 * far:.2f}% away (norm) from those of the sequences")
