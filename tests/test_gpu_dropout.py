"""Dropout and drop path from the keyed draws: which values are kept is checked exactly against the definition
(train_reference.py), the values up to two fp32 roundings and the one to their type."""
import numpy as np
import pytest
import torch

import paper_2404_00509_amd as mae
from train_reference import U32, check, dropout_keep, rounding

pytestmark = pytest.mark.gpu

F32, BF16 = torch.float32, torch.bfloat16


def _inputs(seed, M, D, dtype):
    rng = np.random.default_rng([seed, M, D])
    return tuple(torch.from_numpy(rng.normal(size=(M, D)).astype(np.float32)).to(dtype).cuda() for _ in range(2))


def _check(x, residual, key, y, what):
    keep = torch.from_numpy(np.ascontiguousarray(dropout_keep(*x.shape, **key))).cuda()
    p = float(np.float32(key["p"]))
    scaled = x.double() / (1.0 - p) if p < 1.0 else torch.zeros_like(x, dtype=torch.float64)
    r = torch.zeros_like(scaled) if residual is None else residual.double()
    want = torch.where(keep, scaled, 0.0) + r
    check(y, want, 4 * U32 * (scaled.abs() + r.abs()) + rounding(x.dtype) * 1.01 * want.abs(), what)
    assert torch.equal(y[~keep].double(), r[~keep]), what
    return keep


def _run(x, residual, y=None, stream=None, **key):
    y = torch.full_like(x, float("nan")) if y is None else y
    mae.mae_dropout(mae.make_dropout_desc(x, residual, **key), y, stream=stream)
    return y


SHAPES = [(1, 1), (1, 2), (3, 5), (7, 8), (197, 192), (50, 768), (33, 1017), (4097, 3), (1, 8192), (300, 1024)]


@pytest.mark.parametrize("M,D", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows_per_draw", [0, 1, 3, 197])
def test_values_and_what_is_kept(M, D, dtype, rows_per_draw):
    x, residual = _inputs(1, M, D, dtype)
    for row_base, p in ((0, 0.1), (5, 0.5), (2 ** 33 + 1, 0.25)):  # odd first indices, indices past 32 bits
        key = dict(p=p, rows_per_draw=rows_per_draw, seed=2 ** 63 + 17, batch_index=3, layer=2 ** 31 + 5,
                   row_base=row_base)
        _check(x, residual, key, _run(x, residual, **key), "with residual")
        _check(x, None, key, _run(x, None, **key), "alone")


@pytest.mark.parametrize("rows_per_draw", [0, 4])
def test_ends_of_the_probability(rows_per_draw):
    x, residual = _inputs(2, 40, 96, F32)
    assert torch.equal(_run(x, None, p=0.0, rows_per_draw=rows_per_draw), x)
    assert torch.equal(_run(x, residual, p=1.0, rows_per_draw=rows_per_draw), residual)
    assert not _run(x, None, p=1.0, rows_per_draw=rows_per_draw).any()
    key = dict(p=1e-9, rows_per_draw=rows_per_draw, seed=1, batch_index=1, layer=0, row_base=0)
    _check(x, None, key, _run(x, None, **key), "tiny p")


def test_share_of_dropped_values():
    M, D, p = 4000, 500, 0.3
    y = _run(torch.ones(M, D, device="cuda"), None, p=p, seed=9, batch_index=4, layer=1)
    n = M * D
    assert abs(float((y == 0).double().mean()) - p) < 6 * (p * (1 - p) / n) ** 0.5
    rows = _run(torch.ones(20000, 8, device="cuda"), None, p=p, rows_per_draw=2, seed=9, batch_index=4, layer=1)
    groups = (rows.reshape(10000, 16) == 0).sum(1)
    assert bool(((groups == 0) | (groups == 16)).all())
    assert abs(float((groups == 16).double().mean()) - p) < 6 * (p * (1 - p) / 10000) ** 0.5


def test_other_keys_give_other_draws():
    x = torch.ones(64, 256, device="cuda")
    base = dict(p=0.5, seed=1, batch_index=2, layer=3)
    first = _run(x, None, **base)
    assert torch.equal(first, _run(x, None, **base))
    for change in (dict(seed=2), dict(batch_index=3), dict(layer=4), dict(row_base=64)):
        other = _run(x, None, **{**base, **change})
        assert 0.4 < float((other != first).double().mean()) < 0.6, change


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows_per_draw", [0, 7])
def test_a_split_batch_gives_the_values_of_the_whole(dtype, rows_per_draw):
    M, D = 35, 121
    x, residual = _inputs(3, M, D, dtype)
    key = dict(p=0.4, rows_per_draw=rows_per_draw, seed=5, batch_index=6, layer=7)
    whole = _run(x, residual, **key)
    for cut in (1, 8, 20):
        parts = [_run(x[a:b].clone(), residual[a:b].clone(), row_base=a, **key) for a, b in ((0, cut), (cut, M))]
        assert torch.equal(torch.cat(parts), whole), cut


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows_per_draw", [0, 5])
def test_what_is_dropped_is_not_used(dtype, rows_per_draw):
    M, D = 64, 203
    x, residual = _inputs(4, M, D, dtype)
    key = dict(p=0.5, rows_per_draw=rows_per_draw, seed=1, batch_index=0, layer=0, row_base=0)
    keep = torch.from_numpy(np.ascontiguousarray(dropout_keep(M, D, **key))).cuda()
    for poison in (float("nan"), float("inf")):
        bad = torch.where(keep, x, torch.full_like(x, poison))
        assert torch.equal(_run(bad, residual, **key), _run(x, residual, **key))


@pytest.mark.parametrize("rows_per_draw", [0, 6])
def test_backward_is_the_same_call(rows_per_draw):
    # y is linear in x: a difference of any size is the gradient's product with it
    M, D = 54, 77
    x, d = _inputs(5, M, D, F32)
    g, residual = _inputs(6, M, D, F32)
    key = dict(p=0.2, rows_per_draw=rows_per_draw, seed=11, batch_index=12, layer=13)
    gx = _run(g, None, **key)
    diff = (_run(x + d, residual, **key).double() - _run(x, residual, **key).double()) * g.double()
    size = (x.double().abs() + d.double().abs() + residual.double().abs()) * g.double().abs() * 2
    check((gx.double() * d.double()).sum().reshape(1), diff.sum().reshape(1), 8 * U32 * size.sum(), "inner products")


@pytest.mark.parametrize("rows_per_draw", [0, 3])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_in_place_and_nothing_behind_the_end(dtype, rows_per_draw):
    M, D = 13, 999
    x, residual = _inputs(7, M, D, dtype)
    key = dict(p=0.3, rows_per_draw=rows_per_draw, seed=3)
    want = _run(x, residual, **key)
    xx, rr = x.clone(), residual.clone()
    assert torch.equal(_run(xx, residual, y=xx, **key), want)
    assert torch.equal(_run(x, rr, y=rr, **key), want)
    room = torch.full((M * D + 64,), 5.0, dtype=dtype, device="cuda")
    _run(x, residual, y=room, **key)
    assert torch.equal(room[:M * D].reshape(M, D), want) and bool((room[M * D:] == 5.0).all())


def test_many_values():
    M, D = 70001, 1025  # indices past the grid's first pass; odd rows
    x = torch.ones(M, D, dtype=BF16, device="cuda")
    key = dict(p=0.1, seed=3, batch_index=1, layer=2)
    y = _run(x, None, **key)
    for a, b in ((0, 300), (35000, 35200), (M - 300, M)):
        part = _run(x[a:b].contiguous(), None, row_base=a, **key)
        assert torch.equal(part, y[a:b])
        _check(x[a:b], None, dict(rows_per_draw=0, row_base=a, **key), part, f"rows {a}")


@pytest.mark.parametrize("rows_per_draw", [0, 3])
def test_offsets_past_32_bits(rows_per_draw):
    M, D = 1_060_003, 2053  # more than 2^31 values and 2^32 bytes
    x = torch.ones(M, D, dtype=BF16, device="cuda")
    key = dict(p=0.1, rows_per_draw=rows_per_draw, seed=3, batch_index=1, layer=2)
    y = _run(x, None, **key)
    for a, b in ((0, 99), (1_046_000, 1_046_100), (M - 99, M)):
        _check(x[a:b], None, dict(row_base=a, **key), y[a:b], f"rows {a}")


def test_side_stream_and_replays_of_a_graph():
    x, residual = _inputs(8, 500, 768, BF16)
    key = dict(p=0.1, seed=21, batch_index=22, layer=23)
    want = [_run(x, residual, **key), _run(x, residual, rows_per_draw=50, **key)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _run(x, residual, stream=side, **key)
    side.synchronize()
    assert torch.equal(got, want[0])
    out = [torch.empty_like(x) for _ in range(2)]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s = torch.cuda.current_stream()
        _run(x, residual, y=out[0], stream=s, **key)
        _run(x, residual, y=out[1], stream=s, rows_per_draw=50, **key)
    for k in range(3):
        for t in out:
            t.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k
        x.mul_(1.0)
