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


def _rows_of_a_lane(M, D, ws_bytes):
    """Rows that one lane adds up: the workgroups of the workspace's partial sums, their groups of lanes, one or two rows
    of a group at a time."""
    workgroups = ws_bytes // (8 * (-(-D // 4) * 4))
    lanes = 16 if D <= 384 else 64 if D <= 1536 else 256 if D <= 6144 else 512
    at_once = 2 if lanes <= 64 and -(-D // 4) <= 3 * lanes else 1
    groups = max(256, lanes) // lanes
    return -(-M // (workgroups * groups * at_once)) * at_once


@pytest.mark.parametrize("M,D", [(1, 768), (37, 384), (8191, 48), (40000, 16), (20011, 192), (30001, 385), (9001, 768),
                                 (5003, 2052), (3001, 6145), (60000, 1537), (150001, 100)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_sums_over_rows(M, D, dtype):
    x, gy, w, b = _randn(M + D, (M, D), (M, D), (D,), (D,))
    x, gy = (x + 0.5).to(dtype), gy.to(dtype)
    (_, mean, rstd), grads, ws_bytes = _forward_and_back(x, gy, w, b, 1e-6)
    ref, err = layer_norm_grad(x, gy, w, mean, rstd, _rows_of_a_lane(M, D, ws_bytes))
    for name, got, r, e, t in zip(("grad_x", "grad_weight", "grad_bias"), grads, ref, err, (dtype, F32, F32)):
        check(got, r, e + rounding(t) * (r.abs() + e), name)


def test_sums_of_rows_that_need_every_bit():
    # whole numbers: a workgroup's share of the rows is exact in fp32, and the shares are added in double precision; one fp32
    # sum over all rows would pass 2^24 and lose odd ones
    M, D = 50000, 64
    x = torch.zeros(M, D, device="cuda")
    x[:, ::2], x[:, 1::2] = 1.0, -1.0  # mean 0, h = +-1 with eps = 0
    gy = torch.full((M, D), 4097.0, device="cuda")
    desc = mae.make_norm_desc(x, eps=0.0)
    mean, rstd = torch.zeros(M, device="cuda"), torch.ones(M, device="cuda")
    gw, gb = torch.empty(D, device="cuda"), torch.empty(D, device="cuda")
    ws = torch.empty(mae.mae_layer_norm_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    mae.mae_layer_norm_grad(desc, gy, mean, rstd, None, gw, gb, ws)
    want = torch.full((D,), float(np.float32(4097.0 * M)), device="cuda")
    assert torch.equal(gb, want) and torch.equal(gw, want * x[0])
