"""As many streams and rows as the calls take."""
import pytest

MOST = (1 << 31) - 1


def test_turns_of_all_blocks_stay_in_range():
    """The step's loop over streams in the kernel's arithmetic (32 bits, unsigned): from every block's first stream of a
    last turn the next one is past B, also where a signed sum would have wrapped to a negative stream."""
    import numpy as np
    for B in (MOST, MOST - 3, MOST - 262139, 262140, 5):
        blocks = min((B - 1) // 4 + 1, 65535)
        step, last = 4 * blocks, (B - 1) // (4 * blocks) * 4 * blocks
        for block in {0, blocks // 2, blocks - 1}:
            b0 = last + 4 * block
            while b0 < B:
                wrapped = int(np.uint32(b0) + np.uint32(step))  # no carry out of 32 bits
                assert wrapped == b0 + step < 1 << 32 and b0 + 3 < 1 << 32
                b0 = wrapped
            assert b0 >= B


@pytest.mark.gpu
def test_step_of_the_most_streams(cuda_device):
    """2^31 - 1 streams of one channel, nearly all of them idle."""
    import torch
    from paper_1905_00689_gb300 import gated_step
    x, r, i = (torch.full((1, 1), v, dtype=torch.bfloat16, device="cuda") for v in (1.5, 0.25, -0.5))
    decay = torch.tensor([-4.0], device="cuda")
    state = torch.tensor([[1.0], [2.0], [-3.0], [5.0]], device="cuda")
    want = state.clone()
    y4 = gated_step(x.expand(4, 1), r.expand(4, 1), i.expand(4, 1), decay, want)
    slots = torch.full((MOST,), -1, dtype=torch.int32, device="cuda")
    at = torch.tensor([0, 262140, MOST - 2, MOST - 1], device="cuda")
    slots[at] = torch.arange(4, dtype=torch.int32, device="cuda")
    y = torch.full((MOST, 1), 7.0, dtype=torch.bfloat16, device="cuda")
    gated_step(x.expand(MOST, 1), r.expand(MOST, 1), i.expand(MOST, 1), decay, state, slots=slots, y=y)
    assert torch.equal(state, want) and torch.equal(y[at], y4)
    y[at] = 0.0
    assert int(torch.count_nonzero(y)) == 0


@pytest.mark.gpu
def test_step_of_the_most_channels(cuda_device):
    """One stream of 2^31 - 256 channels: the bits of its pieces."""
    import torch
    from paper_1905_00689_gb300 import gated_step
    D = (1 << 31) - 256
    x = torch.empty(1, D, dtype=torch.bfloat16, device="cuda").normal_()
    decay = torch.empty(D, device="cuda").uniform_(-6.0, -4.0)
    state = torch.ones(1, D, device="cuda")
    y = gated_step(x, x, x, decay, state)
    for at in (0, 1 << 30, D - 4096):
        part, held = x[:, at:at + 4096].contiguous(), torch.ones(1, 4096, device="cuda")
        assert torch.equal(gated_step(part, part, part, decay[at:at + 4096].contiguous(), held), y[:, at:at + 4096])
        assert torch.equal(held, state[:, at:at + 4096])


@pytest.mark.gpu
@pytest.mark.parametrize("K,scale", [(20, "float16"), (40, "float32")])
def test_matvec_of_the_most_rows(cuda_device, K, scale):
    """A matrix of 2^31 - 1 rows, zeros but for a few at both ends (69 GB at 64 columns' pitch)."""
    import torch
    from paper_1905_00689_gb300 import W4Weight, w4_matvec
    N, pitch, G = MOST, -(-K // 32) * 16, -(-K // 32)
    x = torch.randn(2, K, device="cuda").to(torch.bfloat16)
    gen = torch.Generator(device="cuda").manual_seed(3)
    few = torch.randint(0, 256, (300, pitch), generator=gen, device="cuda", dtype=torch.uint8)
    q = torch.full((N, pitch), 0x88, dtype=torch.uint8, device="cuda")  # the zero point of 8: all zeros
    q[:150], q[N - 150:] = few[:150], few[150:]
    s = torch.ones(N, G, dtype=getattr(torch, scale), device="cuda")
    y = w4_matvec(x[:1], W4Weight(q, s, None, K, 32))
    want = w4_matvec(x[:1], W4Weight(few, s[:300].clone(), None, K, 32))
    assert torch.equal(y[:, :150], want[:, :150]) and torch.equal(y[:, N - 150:], want[:, 150:])
    y[:, :150], y[:, N - 150:] = 0.0, 0.0
    assert int(torch.count_nonzero(y)) == 0
    del y
    y = w4_matvec(x, W4Weight(q[N - 300:], s[:300].clone(), None, K, 32))
    assert torch.equal(y[:, 150:], w4_matvec(x, W4Weight(few, s[:300].clone(), None, K, 32))[:, 150:])
