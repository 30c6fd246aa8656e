"""The delta rule where a block has 32 columns of the state (more heads than the device takes at 16): first states, gradients of
the last, lengths and resets, against 64 bits."""
import pytest

import delta_reference as delta
from test_operators_delta_scan import compare_backward, compare_forward, lengths_and_resets


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", [(130, 20, 4, 2, 128, 50), (200, 39, 2, 2, 64, 33), (65, 160, 1, 1, 100, 32), (129, 20, 2, 1, 33, 96)])
def test_masked_and_resumed(cuda_device, dtype, T, B, H, Hk, Dk, Dv):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    assert B * H * -(-Dv // 16) > 152
    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, T + Dv)
    gen = torch.Generator(device="cuda").manual_seed(Dk)
    h0, dh_last = (torch.randn(B, H, Dk, Dv, generator=gen, device="cuda") for _ in range(2))
    do = torch.randn(T, B, H, Dv, generator=gen, device="cuda").to(args[0].dtype)
    lengths, reset = lengths_and_resets(T, B, T + Dk)
    lengths[:4] = torch.tensor([T, T, T - 1, 0], dtype=torch.int32)
    reset[:, 1] = False
    reset[64 - 1, 2] = reset[min(64 + 40, T - 2), 2] = True
    more = dict(lengths=lengths, reset=reset)
    states = delta_scan_states(args[0], args[2])
    states.fill_(float("nan"))
    o, last = delta_scan(*args, h0, states=states, **more)
    grads = delta_scan_backward(do, *args, states, dh_last, **more)
    assert all(torch.isfinite(x.float()).all() for x in (o, last, *grads))
    for some in (slice(0, 4), slice(B - 2, B)):  # the others are in the blocks before and behind
        part = [t[:, some] for t in args]
        cut = dict(h0=h0[some], lengths=lengths[some], reset=reset[:, some])
        compare_forward(part, (o[:, some], last[some]), dtype, **cut)
        compare_backward(do[:, some], part, [x[:, some] for x in grads[:5]] + [grads[5][some]], dtype, dh_last=dh_last[some], **cut)
    plain = delta_scan(*args)  # without any of it
    compare_forward([t[:, B - 1:] for t in args], (plain[0][:, B - 1:], plain[1][B - 1:]), dtype)
