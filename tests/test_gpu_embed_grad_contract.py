"""Gradients of the patch embedding where the interface promises more than sums: infinities and NaN stay in their
position, and which bits do not depend on the outputs that a call asks for."""
import itertools

import pytest
import torch

import paper_2404_00509_amd as mae

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
U32 = torch.finfo(torch.float32).eps / 2
NAN, INF = float("nan"), float("inf")


def _whole(seed, M, D, E, L, most=3):
    g = torch.Generator(device="cuda").manual_seed(seed * 7919 + M + D + E)
    r = lambda *s: torch.randint(-most, most + 1, s, generator=g, device="cuda").to(BF16)  # noqa: E731
    return r(M, D), r(M, E), torch.randint(0, L, (M,), generator=g, device="cuda", dtype=torch.int32)


def _run(visible, g, ids, L, want=(True, True, True)):
    E, D = g.shape[-1], visible.shape[-1]
    w = torch.zeros(E, D, dtype=BF16, device="cuda")  # not read
    pos = None if ids is None else torch.zeros(L, E, device="cuda")
    desc = mae.make_embed_desc(visible, ids, w, None, pos)
    ws = torch.full((mae.mae_patch_embed_grad_workspace_bytes(desc),), 0xFF, dtype=torch.uint8, device="cuda")
    out = [torch.full(s, 7.0, device="cuda") if on else None for on, s in zip(want, ((E, D), (E,), (L, E)))]
    mae.mae_patch_embed_grad(desc, g, *out, ws)
    torch.cuda.synchronize()
    return out


def _same(got, want, what):
    """Whole numbers, infinities and NaN: equal, NaN where NaN."""
    got = got.double().cpu()
    bad = ~((got == want) | (torch.isnan(got) & torch.isnan(want)))
    assert not bool(bad.any()), (what, int(bad.sum()), got[bad][:4], want[bad][:4])


def _plain(visible, g, ids, L):
    """On the CPU, in 64 bits."""
    v, gd = visible.double().cpu(), g.double().cpu()
    pos = torch.zeros(L, g.shape[-1], dtype=torch.float64).index_add_(0, ids.clamp(0, L - 1).long().cpu(), gd)
    return gd.T.contiguous() @ v, gd.sum(0), pos


# tiles of 64, 128 and 256; one and several parts of the sum; widths that make the last row one apart (no multiple of 8);
# positions in one tile, in several, one alone; widths that are copied into padded rows (no multiple of 4)
SIZES = [(70, 64, 64, 16), (300, 12, 36, 5), (129, 588, 100, 70), (2, 8, 8, 4), (513, 100, 70, 49), (900, 768, 768, 196),
         (6300, 256, 512, 300), (20000, 768, 768, 196), (1500, 40, 8, 1), (3000, 8, 40, 1000), (64, 16, 3, 2)]


@pytest.mark.parametrize("M,D,E,L", SIZES)
def test_infinities_and_nan_stay_in_their_position(M, D, E, L):
    visible, g, ids = _whole(1, M, D, E, L)
    if L > 2:
        ids = torch.where(ids == L // 2, ids - 1, ids)  # a patch that no token names
    rng = torch.Generator().manual_seed(M)
    places = [(0, 0, INF), (M - 1, E - 1, -INF), (M - 1, 0, NAN), (M // 2, E // 2, -INF)]
    for v in (INF, -INF, NAN, INF):  # some columns get several, of one sign, of both
        m, e = (int(torch.randint(0, n, (1,), generator=rng)) for n in (M, E))
        places += [(m, e, v), ((m * 7 + 3) % M, e, INF)]
    for m, e, v in places:
        g[m, e] = v
    for got, want, name in zip(_run(visible, g, ids, L), _plain(visible, g, ids, L), ("weight", "bias", "pos")):
        _same(got, want, name)


@pytest.mark.parametrize("D,E", [(64, 64), (588, 100), (768, 768)])
def test_one_infinity_changes_one_position(D, E):
    M, L = 700, 196
    visible, g, ids = _whole(2, M, D, E, L)
    clean = _run(visible, g, ids, L)
    for m in (5, 650, M - 1):  # the last row is joined apart where widths are no multiples of 8
        for value in (INF, -INF, NAN):
            bad = g.clone()
            bad[m, 3] = value
            _, bias, pos = _run(visible, bad, ids, L)
            changed = pos != clean[2]
            assert int(changed.sum()) == 1 and bool(changed[int(ids[m]), 3]), (m, value)
            _same(pos[int(ids[m]), 3], torch.tensor(value, dtype=torch.float64), (m, value))
            _same(bias[3], torch.tensor(value, dtype=torch.float64), (m, value))
            rest = torch.arange(E, device="cuda") != 3
            assert torch.equal(bias[rest], clean[1][rest]), (m, value)


def test_a_whole_gradient_that_is_not_finite():
    M, D, E, L = 5000, 64, 384, 100
    visible, g, ids = _whole(3, M, D, E, L)
    ids = ids // 2 * 2
    _, bias, pos = _run(visible, torch.full_like(g, NAN), ids, L)
    assert torch.isnan(bias).all() and torch.isnan(pos[::2]).all() and not pos[1::2].any()
    half = torch.where((ids % 4 == 0)[:, None], torch.full_like(g, INF), g)
    for got, want, name in zip(_run(visible, half, ids, L)[1:], _plain(visible, half, ids, L)[1:], ("bias", "pos")):
        _same(got, want, name)


@pytest.mark.parametrize("M,D,E,L", [(3000, 588, 384, 64), (3000, 588, 70, 64), (3001, 12, 36, 300), (500, 64, 64, 16),
                                     (30000, 768, 768, 196), (2500, 100, 70, 1)])
def test_bits_and_what_else_is_asked_for(M, D, E, L):
    g = torch.Generator(device="cuda").manual_seed(M + E)
    visible = torch.randn(M, D, generator=g, device="cuda").to(BF16)
    grad = torch.randn(M, E, generator=g, device="cuda").to(BF16)
    ids = torch.randint(0, L, (M,), generator=g, device="cuda", dtype=torch.int32)
    whole = _run(visible, grad, ids, L)
    alone = _run(visible, grad, ids, L, (False, True, False))[1]
    for want in itertools.product((False, True), repeat=3):
        if any(want):
            weight, bias, pos = _run(visible, grad, ids, L, want)
            assert weight is None or torch.equal(weight, whole[0]), want
            assert pos is None or torch.equal(pos, whole[2]), want
            # the bias by positions, or in one sum without them
            assert bias is None or torch.equal(bias, whole[1] if want[2] else alone), want
    double = whole[2].double()
    exact, size = grad.double().sum(0), grad.double().abs().sum(0)
    # (64 sums of L / 64 in 64 bits each: at most half a step of fp32, and one of its double)
    assert bool(((whole[1].double() - double.sum(0)).abs() <= U32 * (1 + 1e-6) * double.abs().sum(0)).all())
    for bias in (whole[1], alone):  # M roundings of fp32 sums, one of the result
        assert bool(((bias.double() - exact).abs() <= (M + 1) * U32 * size).all())
    none = _run(visible, grad, None, L, (True, True, False))  # an embedding without positional rows
    for want in ((True, False, False), (False, True, False)):
        for a, b in zip(_run(visible, grad, None, L, want), none):
            assert a is None or torch.equal(a, b), want


def test_weight_and_bias_in_replays_of_a_graph():
    M, D, E, L = 2500, 768, 384, 196
    visible, g, ids = _whole(4, M, D, E, L)
    want = _run(visible, g, ids, L, (True, True, False))
    weight, pos = torch.zeros(E, D, dtype=BF16, device="cuda"), torch.zeros(L, E, device="cuda")
    desc = mae.make_embed_desc(visible, ids, weight, None, pos)
    ws = torch.empty(mae.mae_patch_embed_grad_workspace_bytes(desc), dtype=torch.uint8, device="cuda")
    out = [torch.empty_like(t) for t in want[:2]]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mae.mae_patch_embed_grad(desc, g, *out, None, ws, stream=torch.cuda.current_stream())
    for k in range(3):
        for t in out:
            t.fill_(NAN)
        ws.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want)), k
