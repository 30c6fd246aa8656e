"""Tensors without rows, with the empty axis in any place."""
import pytest


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(0,), (3, 0), (0, 3), (3, 0, 2), (2, 3, 0)])
def test_no_rows(cuda_device, lead):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward, rms_norm_quant, w4_matvec, w4_quantize
    w = torch.ones(64, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        x, rstd = torch.empty(*lead, 64, device="cuda", dtype=dtype), torch.empty(*lead, device="cuda")
        y, _ = rms_norm(x, w, rstd=rstd)
        assert y.shape == x.shape and y.dtype == dtype
        q, scales, _ = rms_norm_quant(x, w, group=32)
        assert q.shape == x.shape and scales.shape == (*lead, 2)
        dx, dw = rms_norm_backward(x, x, w, rstd, x)
        assert dx.shape == x.shape and bool((dw == 0).all())
        W = w4_quantize(torch.randn(5, 64, device="cuda"), 32)
        assert w4_matvec(x, W, bias=torch.ones(5, device="cuda")).shape == (*lead, 5)
        wide = torch.empty(*lead, 200, device="cuda", dtype=dtype)[..., 7:71]
        assert rms_norm(wide, w)[0].shape == x.shape


@pytest.mark.gpu
@pytest.mark.parametrize("lead", [(0,), (3, 0)])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_sum_of_no_rows(cuda_device, lead, dtype):
    """A residual without rows has a sum without rows, not none."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward, rms_norm_quant
    w = torch.ones(64, device="cuda")
    x, rstd = torch.empty(*lead, 64, device="cuda", dtype=getattr(torch, dtype)), torch.empty(*lead, device="cuda")
    y, total = rms_norm(x, w, x.clone(), rstd=rstd)
    assert y.shape == total.shape == x.shape and total.dtype == x.dtype
    dx, dw = rms_norm_backward(x, total, w, rstd, x)
    assert dx.shape == x.shape and bool((dw == 0).all())
    assert rms_norm_quant(x, w, x.clone())[2].shape == x.shape
