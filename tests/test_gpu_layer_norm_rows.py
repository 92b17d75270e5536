"""Layer norm's backward pass: rows of one large value at widths that leave lanes without values, and sums over rows
with bounds from the geometry that runs."""
import numpy as np
import pytest
import torch

import paper_2404_00509_amd as mae
from train_reference import U32, check, layer_norm_grad, rounding

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _randn(seed, *shapes):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randn(*s, generator=g, device="cuda") for s in shapes]


def _forward_and_back(x, gy, w, b, eps):
    desc = mae.make_norm_desc(x, w, b, eps=eps)
    nan = lambda *s, dtype=F32: torch.full(s, float("nan"), dtype=dtype, device="cuda")  # noqa: E731
    y, mean, rstd = nan(*x.shape, dtype=x.dtype), nan(desc.M), nan(desc.M)
    mae.mae_layer_norm(desc, y, mean, rstd)
    grads = nan(*x.shape, dtype=x.dtype), nan(desc.D), nan(desc.D)
    ws = torch.full((mae.mae_layer_norm_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    mae.mae_layer_norm_grad(desc, gy, mean, rstd, *grads, ws)
    torch.cuda.synchronize()
    return (y, mean, rstd), grads, ws.numel()


# 16 lanes, a wavefront, workgroups of 256 and 512 per row
@pytest.mark.parametrize("D", [1, 2, 3, 6, 7, 8, 33, 100, 385, 588, 1017, 1532, 2045, 6143, 6147, 8190])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_rows_of_one_large_value(D, dtype):
    M, value = 37, 2.0 ** 110
    gy, w, b = _randn(D, (M, D), (D,), (D,))
    gy = gy.to(dtype)
    x = torch.full((M, D), value, dtype=dtype, device="cuda")
    x[::2] = -value
    # sums of up to 8192 of them are exact: h is 0, and 1 / sqrt(eps) = 10^6 times the value is no float
    (y, mean, rstd), grads, _ = _forward_and_back(x, gy, w, b, 1e-12)
    assert torch.equal(mean, x[:, 0].float()) and torch.equal(y, b.expand(M, D).to(dtype))
    assert bool(((rstd.double() * 1e-6 - 1).abs() < 1e-6).all())
    ref, err = layer_norm_grad(x, gy, w, mean, rstd, M)
    for name, got, r, e, t in zip(("grad_x", "grad_weight", "grad_bias"), grads, ref, err, (dtype, F32, F32)):
        check(got, r, e + rounding(t) * (r.abs() + e), name)
