"""The operators record nothing for torch's differentiation, as documented: gradients are calls of their own."""
import pytest


@pytest.mark.gpu
def test_outputs_have_no_history(cuda_device):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_step, rms_norm, w4_matvec, w4_quantize
    x = torch.randn(3, 2, 64, device="cuda", requires_grad=True)
    w = torch.ones(64, device="cuda", requires_grad=True)
    decay = torch.full((64,), -5.0, device="cuda", requires_grad=True)
    outs = [*rms_norm(x, w, x), *gated_scan(x, x, x, decay), gated_step(x[0], x[0], x[0], decay, torch.zeros(2, 64, device="cuda")),
            w4_matvec(x, w4_quantize(torch.randn(5, 64, device="cuda", requires_grad=True)))]
    assert all(not t.requires_grad and t.grad_fn is None for t in outs)
    with torch.no_grad():
        assert torch.equal(outs[0], rms_norm(x, w, x)[0])
