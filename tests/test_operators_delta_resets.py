"""A reset's own decay takes part in nothing, in a step as in a sequence."""
import pytest

import delta_reference as delta


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf"), 90.0])
@pytest.mark.parametrize("dtype,Dk,Dv", [("fp32", 64, 32), ("bf16", 128, 50)])
def test_the_decay_of_a_reset_may_be_anything(cuda_device, dtype, Dk, Dv, value):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states, delta_step
    B, H, Hk, T = 3, 2, 1, 70
    q, k, v, g, beta = delta.tensors((B,), H, Hk, Dk, Dv, dtype, 2)
    held = torch.randn(B, H, Dk, Dv, device="cuda")
    held[1] = float("nan")
    reset = torch.tensor([False, True, True], device="cuda")
    results = []
    for at in (0.0, value):
        state, gates = held.clone(), g.clone()
        gates[reset] = at
        results.append((delta_step(q, k, v, gates, beta, state, reset=reset), state))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and torch.isfinite(results[0][1]).all()

    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, 3)
    cuts = torch.zeros(T, B, dtype=torch.bool, device="cuda")
    cuts[0, 1] = cuts[33, 0] = cuts[64, 2] = True
    do, results = torch.randn(T, B, H, Dv, device="cuda").to(args[2].dtype), []
    for at in (0.0, value):
        gates, states = args[3].clone(), delta_scan_states(args[0], args[2])
        gates[cuts] = at
        call = (*args[:3], gates, args[4])
        out = delta_scan(*call, held, reset=cuts, states=states)
        results.append((*out, *delta_scan_backward(do, *call, states, reset=cuts)))
    assert all(torch.equal(a, b) for a, b in zip(*results)) and all(torch.isfinite(x.float()).all() for x in results[0])
