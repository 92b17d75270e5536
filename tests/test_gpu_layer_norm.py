"""Layer norm and its backward pass against the formulas in 64 bits, with bounds from fp32 arithmetic
(train_reference.py): every kernel variant (16 lanes, a wavefront, a workgroup per row), widths that are no multiple
of four, one row, all pairs of types, tensors on no 16-byte boundary, work in place."""
import numpy as np
import pytest
import torch

import paper_2404_00509_amd as mae
from train_reference import U32, check, layer_norm, layer_norm_grad, rounding

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16
MAE_DTYPE = {F32: mae.MAE_F32, BF16: mae.MAE_BF16}
TYPES = [(F32, F32), (BF16, BF16), (BF16, F32), (F32, BF16)]


def _inputs(seed, M, D, x_type, y_type, affine=True):
    rng = np.random.default_rng([seed, M, D])
    t = lambda *s: torch.from_numpy(rng.normal(size=s).astype(np.float32)).cuda()  # noqa: E731
    x = (t(M, D) * (0.5 + t(M, 1).abs()) + t(M, 1) + 0.5 * t(1, D)).to(x_type)
    gy = t(M, D).to(y_type)
    return x, gy, (1 + 0.2 * t(D)) if affine else None, t(D) if affine else None


def _forward(x, w, b, eps, y_type, stream=None):
    desc = mae.make_norm_desc(x, w, b, eps=eps, y_dtype=MAE_DTYPE[y_type])
    y = torch.full(x.shape, float("nan"), dtype=y_type, device="cuda")
    mean, rstd = (torch.full((desc.M,), float("nan"), device="cuda") for _ in range(2))
    mae.mae_layer_norm(desc, y, mean, rstd, stream=stream)
    return desc, y, mean, rstd


def _workspace(desc):
    return torch.full((max(mae.mae_layer_norm_workspace_bytes(desc), 256),), 0xFF, dtype=torch.uint8, device="cuda")


def _backward(desc, x, gy, mean, rstd, want=(True, True, True), stream=None):
    out = [torch.full(s, float("nan"), dtype=t, device="cuda") if on else None
           for on, s, t in zip(want, (x.shape, (desc.D,), (desc.D,)), (x.dtype, F32, F32))]
    mae.mae_layer_norm_grad(desc, gy, mean, rstd, *out, _workspace(desc), stream=stream)
    return out


def _rows_in_turn(M, D):
    at_once = 1024 * (16 if D <= 64 else 4 if D <= 2048 else 1)
    return -(-M // at_once)


def _check_all(x, gy, w, b, eps, y_type, what):
    desc, y, mean, rstd = _forward(x, w, b, eps, y_type)
    (ry, rmean, rrstd), (ey, emean, erstd) = layer_norm(x, w, b, eps)
    check(mean, rmean, emean + U32 * rmean.abs(), what + " mean")
    check(rstd, rrstd, erstd, what + " rstd")
    check(y, ry, ey + rounding(y_type) * (ry.abs() + ey), what + " y")
    grads = _backward(desc, x, gy, mean, rstd)
    ref, err = layer_norm_grad(x, gy, w, mean, rstd, _rows_in_turn(*x.shape))
    kinds = (x.dtype, F32, F32)
    for name, got, r, e, t in zip(("grad_x", "grad_weight", "grad_bias"), grads, ref, err, kinds):
        check(got, r, e + rounding(t) * (r.abs() + e), f"{what} {name}")


WIDTHS = [1, 2, 3, 4, 7, 16, 63, 64, 65, 100, 192, 255, 256, 257, 384, 588, 768, 1017, 1024, 1280, 1536, 2045, 2048,
          2049, 3071, 4096, 5003, 6148, 8191, 8192]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("x_type,y_type", TYPES)
def test_widths_and_types(D, x_type, y_type):
    for M in (1, 37):
        x, gy, w, b = _inputs(1, M, D, x_type, y_type)
        _check_all(x, gy, w, b, 1e-6, y_type, f"M{M} D{D}")


@pytest.mark.parametrize("M,D", [(1, 768), (2, 768), (3, 192), (8191, 48), (40000, 16), (20011, 192), (9001, 768),
                                 (5003, 2052)])
@pytest.mark.parametrize("x_type,y_type", [(BF16, BF16), (F32, F32)])
def test_numbers_of_rows(M, D, x_type, y_type):
    x, gy, w, b = _inputs(2, M, D, x_type, y_type)
    _check_all(x, gy, w, b, 1e-5, y_type, f"M{M} D{D}")


@pytest.mark.parametrize("D", [48, 768, 4096])
def test_without_weight_and_bias(D):
    x, gy, _, _ = _inputs(3, 33, D, F32, F32, affine=False)
    _check_all(x, gy, None, None, 1e-6, F32, "plain")
    w = torch.rand(D, device="cuda") + 0.5
    _check_all(x, gy, w, None, 1e-6, F32, "weight alone")
    _check_all(x, gy, None, w, 1e-6, F32, "bias alone")


@pytest.mark.parametrize("D", [60, 768, 4100])
def test_each_gradient_by_itself(D):
    x, gy, w, b = _inputs(4, 257, D, BF16, BF16)
    desc, _, mean, rstd = _forward(x, w, b, 1e-6, BF16)
    whole = _backward(desc, x, gy, mean, rstd)
    for k in range(3):
        want = [k == i for i in range(3)]
        part = _backward(desc, x, gy, mean, rstd, want)
        assert torch.equal(part[k], whole[k]), k
    # no workspace without the parameters' gradients
    gx = torch.full_like(x, float("nan"))
    mae.mae_layer_norm_grad(desc, gy, mean, rstd, gx)
    assert torch.equal(gx, whole[0])
    y = torch.empty_like(x)
    mae.mae_layer_norm(desc, y)  # no statistics
    assert not torch.isnan(y).any()


def test_constant_rows_and_an_offset_much_larger_than_the_spread():
    x, gy, w, b = _inputs(5, 64, 768, F32, F32)
    x[::2] = 3.0  # variance 0: y = bias
    x[1::2] = 1000.0 + 0.01 * x[1::2]
    _check_all(x, gy, w, b, 1e-6, F32, "offset")
    _, y, _, rstd = _forward(x, w, b, 1e-6, F32)
    assert torch.equal(y[::2], b.expand(32, -1))
    assert torch.equal(rstd[::2], torch.full_like(rstd[::2], float(np.float32(1.0) / np.sqrt(np.float32(1e-6)))))


def test_a_row_that_is_not_finite_stays_alone():
    x, gy, w, b = _inputs(6, 70, 768, F32, F32)
    clean = _forward(x, w, b, 1e-6, F32)[1]
    x[5, 3], x[17, 700], x[69, 0] = float("nan"), float("inf"), -float("inf")
    _, y, _, _ = _forward(x, w, b, 1e-6, F32)
    rest = torch.ones(70, dtype=torch.bool, device="cuda")
    rest[[5, 17, 69]] = False
    assert torch.equal(y[rest], clean[rest])
    assert torch.isnan(y[5]).all() and torch.isnan(y[17]).any() and torch.isnan(y[69]).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("D", [33, 255, 768, 3001])
def test_tensors_on_any_boundary_of_their_values(D, dtype):
    M = 19
    x, gy, w, b = _inputs(7, M, D, dtype, dtype)
    moved = [torch.cat([t.new_zeros(1), t.reshape(-1)])[1:].reshape(t.shape) for t in (x, gy, w, b)]
    assert moved[0].is_contiguous() and moved[0].data_ptr() % 16 != 0
    desc, y, mean, rstd = _forward(x, w, b, 1e-6, dtype)
    desc2, y2, mean2, rstd2 = _forward(moved[0], moved[2], moved[3], 1e-6, dtype)
    assert torch.equal(y, y2) and torch.equal(mean, mean2) and torch.equal(rstd, rstd2)
    out = torch.full((M * D + 1,), float("nan"), dtype=dtype, device="cuda")
    mae.mae_layer_norm(desc2, out[1:])
    assert torch.isnan(out[0]) and torch.equal(out[1:].reshape(M, D), y)
    for got, want in zip(_backward(desc2, moved[0], moved[1], mean, rstd), _backward(desc, x, gy, mean, rstd)):
        assert torch.equal(got, want)


@pytest.mark.parametrize("D", [50, 768, 2500])
def test_in_place_and_nothing_behind_the_last_row(D):
    M = 29
    x, gy, w, b = _inputs(8, M, D, BF16, BF16)
    desc, y, mean, rstd = _forward(x, w, b, 1e-6, BF16)
    gx = _backward(desc, x, gy, mean, rstd)[0]
    room = torch.full((M + 3, D), 7.0, dtype=BF16, device="cuda")
    room[:M] = x
    mae.mae_layer_norm(mae.make_norm_desc(room[:M], w, b), room[:M])
    assert torch.equal(room[:M], y) and bool((room[M:] == 7.0).all())
    for over in ("x", "grad_y"):
        xx, gg = x.clone(), gy.clone()
        mae.mae_layer_norm_grad(mae.make_norm_desc(xx, w, b), gg, mean, rstd, xx if over == "x" else gg)
        assert torch.equal(xx if over == "x" else gg, gx), over


def test_offsets_past_32_bits():
    M, D = 1_060_003, 2053  # more than 2^31 values and 2^32 bytes
    base = _inputs(11, 1009, D, BF16, BF16)
    x, gy = (t.repeat(M // 1009 + 1, 1)[:M].contiguous() for t in base[:2])
    w, b = base[2:]
    desc, y, mean, rstd = _forward(x, w, b, 1e-6, BF16)
    gx, gw, gb = _backward(desc, x, gy, mean, rstd)
    _, y1, mean1, rstd1 = _forward(*base[:1], w, b, 1e-6, BF16)
    gx1 = _backward(mae.make_norm_desc(base[0], w, b), base[0], base[1], mean1, rstd1)[0]
    for at in (0, 1009 * 500, 1009 * 1049):
        assert torch.equal(y[at:at + 1009], y1) and torch.equal(gx[at:at + 1009], gx1)
        assert torch.equal(mean[at:at + 1009], mean1) and torch.equal(rstd[at:at + 1009], rstd1)
    tail = M % 1009
    assert torch.equal(y[M - tail:], y1[:tail]) and torch.equal(gx[M - tail:], gx1[:tail])
    h = (base[0].double() - mean1.double()[:, None]) * rstd1.double()[:, None]
    times = torch.full((1009, 1), float(M // 1009), dtype=torch.float64, device="cuda")
    times[:tail] += 1
    n = (_rows_in_turn(M, D) + 12) * U32
    g = base[1].double() * times
    check(gw, (g * h).sum(0), (n + U32) * (g * h).abs().sum(0), "grad_weight")
    check(gb, g.sum(0), (n + U32) * g.abs().sum(0), "grad_bias")


def test_gradient_against_differences():
    M, D, h = 24, 96, 2.0 ** -6
    x, c, w, b = _inputs(9, M, D, F32, F32)
    x = (x * 16).round() / 16  # x + h d and x - h d are exact
    d = torch.where(torch.rand(M, D, device="cuda") < 0.5, -1.0, 1.0)
    desc, _, mean, rstd = _forward(x, w, b, 1e-6, F32)
    gx, gw, gb = _backward(desc, x, c, mean, rstd)
    values, exact = [], []
    for s in (h, -h):
        values.append((_forward(x + s * d, w, b, 1e-6, F32)[1].double() * c.double()).sum(1))
        (y, _, _), (e, _, _) = layer_norm(x + s * d, w, b, 1e-6)
        exact.append((y * c.double()).sum(1))
    slope = (values[0] - values[1]) / (2 * h)
    plain = (exact[0] - exact[1]) / (2 * h)
    noise = ((e + U32 * y.abs()) * c.double().abs()).sum(1) / h
    check(slope, plain, noise * 1.1, "difference quotient")
    (rx, rw, rb), _ = layer_norm_grad(x, c, w, mean, rstd, 1)
    bent = ((rx * d.double()).sum(1) - plain).abs()  # what the difference's curvature makes of it
    assert float(bent.max()) < 0.02 * float((rx * d.double()).sum(1).abs().max())
    check((gx.double() * d.double()).sum(1), slope, noise * 1.1 + bent + 64 * U32 * (rx.abs().sum(1) + 1), "gradient")
    # linear in weight and bias: differences of any size are exact but for rounding
    y1 = _forward(x, w + 1.0, b, 1e-6, F32)[1].double()
    y0 = _forward(x, w, b, 1e-6, F32)[1].double()
    check(gw, ((y1 - y0) * c.double()).sum(0), 16 * U32 * ((y1.abs() + y0.abs()) * c.double().abs()).sum(0), "weight")
    y1 = _forward(x, w, b + 1.0, 1e-6, F32)[1].double()
    check(gb, ((y1 - y0) * c.double()).sum(0), 16 * U32 * ((y1.abs() + y0.abs() + 1) * c.double().abs()).sum(0), "bias")


def test_side_stream_and_replays_of_a_graph():
    M, D = 1500, 768
    x, gy, w, b = _inputs(10, M, D, BF16, BF16)
    desc, y, mean, rstd = _forward(x, w, b, 1e-6, BF16)
    grads = _backward(desc, x, gy, mean, rstd)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        _, y2, _, _ = _forward(x, w, b, 1e-6, BF16, stream=side)
        again = _backward(desc, x, gy, mean, rstd, stream=side)
    side.synchronize()
    assert torch.equal(y, y2) and all(torch.equal(p, q) for p, q in zip(grads, again))
    out = [torch.empty_like(t) for t in (y, mean, rstd, *grads)]
    ws = _workspace(desc)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mae.mae_layer_norm(desc, *out[:3], stream=torch.cuda.current_stream())
        mae.mae_layer_norm_grad(desc, gy, out[1], out[2], *out[3:], ws, stream=torch.cuda.current_stream())
    for k in range(3):
        for t in out:
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for got, want in zip(out, (y, mean, rstd, *grads)):
            assert torch.equal(got, want), k
        x.mul_(1.0)  # eager work between replays
