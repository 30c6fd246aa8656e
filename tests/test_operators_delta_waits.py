"""The delta rule over a sequence where a chunk's copy does not come: the kernels end, with NaN."""
import os
import re

import pytest

import delta_reference as delta
import paper_1905_00689_gb300 as package

CSRC = os.path.join(os.path.dirname(package.__file__), "csrc")


def test_pieces_do_not_go_by_what_a_copy_brings():
    """The loops over a chunk's pieces hold barriers among warps that wait for the copy each by itself.  After a wait that ran out
    the stage may change between two warps' looks at it, so what these loops go by must not lie there (CPU: reads the
    source)."""
    with open(os.path.join(CSRC, "k_delta_scan.cu")) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    for kernel in ("delta_forward_kernel", "delta_backward_kernel"):
        body = text[text.index(f"{kernel}(const DeltaArgs a)"):]
        body = body[:body.index("\n}\n")]
        assert "piece_end(cuts" in body
        assert not re.search(r"gates?\.cuts|gates->cuts", body)


def test_waits_are_checked(lib):
    assert lib.lstm_approx_delta_scan_set_waits(-1, -1) == 1
    assert lib.lstm_approx_delta_scan_set_waits(0, -2) == 1
    assert lib.lstm_approx_delta_scan_set_waits(0, -1) == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,B,Dk,Dv", [("bf16", 2, 128, 40), ("bf16", 30, 64, 100), ("fp32", 2, 128, 24), ("fp16", 3, 33, 17)])
@pytest.mark.parametrize("cut", [False, True])
def test_a_copy_that_does_not_come(cuda_device, lib, dtype, B, Dk, Dv, cut):
    """Chunk 2 of 5 does not come: what does not need it is as ever, what needs it is NaN, and the next call is right.  With
    resets the pieces of that chunk and of the others are as many for all warps."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, H, Hk = 300, 4, 2
    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, 31)
    do = torch.randn(T, B, H, Dv, device="cuda").to(args[0].dtype)
    reset = torch.zeros(T, B, dtype=torch.bool, device="cuda")
    if cut:
        for t in (70, 130, 131, 160, 191, 200, 290):
            reset[t] = True
    more = dict(reset=reset)

    def run():
        states = delta_scan_states(args[0], args[2])
        o, last = delta_scan(*args, states=states, **more)
        return o, last, states
    want = run()
    grads = delta_scan_backward(do, *args, want[2], **more)
    try:
        assert lib.lstm_approx_delta_scan_set_waits(200_000, 2) == 0
        o, last, states = run()
        assert lib.lstm_approx_delta_scan_set_waits(200_000, 2) == 0
        off = delta_scan_backward(do, *args, want[2], **more)
        torch.cuda.synchronize()
    finally:
        assert lib.lstm_approx_delta_scan_set_waits(0, -1) == 0
    assert torch.equal(o[:128], want[0][:128]) and torch.equal(states[:2], want[2][:2])
    assert torch.isnan(o[128:192]).all()
    assert torch.isnan(o[192:]).all() and torch.isnan(last).all()  # (no later copy is waited for)
    dv, dh0 = off[2], off[5]
    assert torch.equal(dv[192:], grads[2][192:])
    assert torch.isnan(dv[:192]).all()
    assert torch.isnan(dh0).all()
    again = run()
    assert all(torch.equal(a, b) for a, b in zip(again[:2], want[:2]))
    assert all(torch.equal(a, b) for a, b in zip(delta_scan_backward(do, *args, again[2], **more), grads))
