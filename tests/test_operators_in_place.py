"""Calls whose outputs lie where their inputs did, as include/lstm_approx_ops.h allows them."""
import numpy as np
import pytest

from test_operators_scan import C, compare_forward, tensors


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,B,D", [(700, 2, 96), (4200, 1, 8), (300, 30, 130), (130, 500, 64)])
def test_last_state_over_the_first(cuda_device, T, B, D, dtype):
    """h_last is h0, over sequences of several tiles: one group of them, several groups, groups of a few and of one
    tile.  The first state is what every tile after it depends on, the last is written by another block."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_states
    x, r, i, decay, _, h0 = tensors(T, B, D, dtype, 300 + T)
    rng = np.random.default_rng(T)
    lengths = torch.tensor(rng.integers(-1, T + 2, B), dtype=torch.int32, device="cuda")
    reset = torch.tensor(rng.random((T, B)) < 0.01, device="cuda")
    reset[0, 0] = True
    for more in ({}, dict(lengths=lengths), dict(lengths=lengths, reset=reset)):
        want_states, states = gated_scan_states(T, B, D), gated_scan_states(T, B, D)
        want = gated_scan(x, r, i, decay, h0, c=C, states=want_states, **more)
        for _ in range(3):
            held = h0.clone()
            y, last = gated_scan(x, r, i, decay, held, c=C, h_last=held, states=states, **more)
            assert last is held and torch.equal(y, want[0]) and torch.equal(held, want[1])
            assert torch.equal(states, want_states)
    if T * B <= 2000:
        held = h0.clone()
        compare_forward((x, r, i, decay), gated_scan(x, r, i, decay, held, c=C, h_last=held), dtype, h0=h0)
