"""Softmax cross entropy of a linear head against the formulas in 64 bits, with bounds from the stated
method (train_reference.py): logits in fp32, the gradient of the logits rounded to fp16 for the two products."""
import numpy as np
import pytest
import torch

import paper_2404_00509_amd as mae
from train_reference import U16, check, class_loss

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16
GRADS = ("grad_tokens", "grad_weight", "grad_bias")


def _inputs(seed, M, D, V, bias=True, left_out=0.0, spread=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed * 1000003 + M * 1009 + D * 31 + V)
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    w = (spread * randn(V, D) / D ** 0.5).to(BF16)
    y = torch.randint(0, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    x = (randn(M, D) + 4 * torch.rand(M, 1, generator=g, device="cuda") * w[y.long()].float()).to(BF16)
    y = torch.where(torch.rand(M, generator=g, device="cuda") < left_out, torch.full_like(y, -1), y)
    return x, y, w, randn(V) if bias else None


def _workspace(desc, grad):
    n = mae.mae_class_loss_workspace_bytes(desc, grad)
    assert n > 0
    return torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")  # (as floats: NaN)


def _run(x, y, w, b, smoothing=0.0, grad_scale=1.0, want=GRADS, ws=None, stream=None):
    desc = mae.make_class_desc(x, y, w, b, smoothing=smoothing, grad_scale=grad_scale)
    nan = float("nan")
    out = {"loss": torch.full((1,), nan, device="cuda"), "row_loss": torch.full((desc.M,), nan, device="cuda")}
    shapes = {"grad_tokens": (x.shape, BF16), "grad_weight": (w.shape, BF16), "grad_bias": ((desc.V,), torch.float32)}
    for k in want:
        if k != "grad_bias" or b is not None:
            out[k] = torch.full(shapes[k][0], nan, dtype=shapes[k][1], device="cuda")
    mae.mae_class_loss(desc, out["loss"], out["row_loss"], *(out.get(k) for k in GRADS),
                       _workspace(desc, bool(want)) if ws is None else ws, stream=stream)
    return out


def _check(x, y, w, b, smoothing=0.0, grad_scale=1.0, what=""):
    out = _run(x, y, w, b, smoothing, grad_scale)
    ref, bound = class_loss(x, y, w, b, smoothing, grad_scale)
    for k, v in out.items():
        check(v, ref[k], bound[k], f"{what} {k}")
    return out


# rows, values, classes: tiles of 64, 128 and 256 classes and rows, whole and ragged ones, one row, one class, sums over
# D of less than a slice of 64, of several, with 8 values behind the last whole slice
SIZES = [(1, 8, 1), (1, 8, 2), (1, 64, 1000), (3, 16, 5), (64, 192, 1000), (65, 72, 64), (63, 200, 65),
         (257, 128, 1003), (300, 328, 2049), (512, 1024, 127), (1000, 64, 3001), (2050, 24, 2000), (4096, 96, 1000),
         (130, 8, 20011), (7, 768, 9001), (4100, 136, 8200), (2049, 192, 16385)]


@pytest.mark.parametrize("M,D,V", SIZES)
def test_sizes(M, D, V):
    for bias, smoothing, left_out in ((True, 0.1, 0.0), (False, 0.0, 0.3)):
        x, y, w, b = _inputs(1, M, D, V, bias, left_out)
        _check(x, y, w, b, smoothing, what=f"M{M} D{D} V{V} bias {bias}")


# without bias and smoothing exponentials are kept for the gradient, else the logits up to 64 MiB and nothing beyond; tiles
# of all sides; the last group of classes whole, ragged and of one class
@pytest.mark.parametrize("M,D,V", [(2048, 64, 8192), (2048, 64, 8193), (16390, 40, 1024), (17000, 8, 1000), (17, 24, 1 << 20),
                                   (200, 72, 90_001), (60, 16, 300_000)])
def test_what_is_kept_for_the_gradient(M, D, V):
    for bias, smoothing, left_out in ((False, 0.0, 0.2), (False, 0.1, 0.0), (True, 0.0, 0.0)):
        x, y, w, b = _inputs(16, M, D, V, bias, left_out, 4.0)
        _check(x, y, w, b, smoothing, -0.5, what=f"M{M} D{D} V{V} bias {bias}")


def test_kept_exponentials_of_far_tiles_and_of_a_row_that_is_not_finite():
    M, D, V = 2100, 64, 8300
    x, y, w, _ = _inputs(17, M, D, V, False, spread=30.0)  # most groups of classes lie far under their row's maximum
    clean = _check(x, y, w, None, what="far")
    x[77, 3] = float("inf")
    out = _run(x, y, w, None)
    rest = torch.arange(M, device="cuda") != 77
    assert torch.isnan(out["loss"]).all() and torch.isnan(out["grad_tokens"][77]).all()
    assert torch.equal(out["row_loss"][rest], clean["row_loss"][rest])
    assert torch.equal(out["grad_tokens"][rest], clean["grad_tokens"][rest])
    none = _run(x, torch.full_like(y, -1), w, None)
    assert not any(bool(v.any()) for v in none.values())


def test_vocabulary_in_pieces_without_a_bias():
    # the first piece from what was kept, the other anew
    M, D, V = 1 << 18, 8, 2100
    x, y, w, b = _inputs(18, M, D, V, False, 0.2)
    _check(x, y, w, b, 0.0, what="pieces")


def test_vocabulary_in_pieces():
    # the gradient goes through the classes 2048 at a time here, and the rows' labels lie in all of them
    M, D, V = 1 << 18, 8, 2100
    x, y, w, b = _inputs(2, M, D, V, True, 0.2)
    _check(x, y, w, b, 0.1, what="pieces")


@pytest.mark.parametrize("smoothing,grad_scale", [(1.0, 1.0), (0.3, -2.5), (0.0, 1024.0), (0.0, 0.0)])
def test_smoothing_and_scale(smoothing, grad_scale):
    x, y, w, b = _inputs(3, 200, 64, 300)
    _check(x, y, w, b, smoothing, grad_scale)


@pytest.mark.parametrize("bias", [False, True])
def test_probabilities_near_the_smoothed_targets(bias):
    # softmax and s / V agree to a few hundredths, and g is what is left of them
    x, y, w, b = _inputs(20, 300, 64, 500, bias, spread=0.02)
    _check(x, y, w, b * 0.02 if bias else None, 1.0, what="near")


@pytest.mark.parametrize("spread", [0.0, 8.0, 60.0])
def test_flat_and_confident_logits(spread):
    x, y, w, b = _inputs(4, 260, 64, 500, spread=spread)
    _check(x, y, w, b, 0.0, what=f"spread {spread}")


def test_rows_that_are_left_out_touch_nothing():
    M, D, V = 700, 128, 900
    x, y, w, b = _inputs(5, M, D, V)
    gone = torch.rand(M, device="cuda") < 0.5
    for label in (-1, V, -2 ** 31, 2 ** 31 - 1):
        yy = torch.where(gone, torch.full_like(y, label), y)
        clean = _run(x, yy, w, b, 0.1)
        for poison in (float("nan"), float("inf"), -float("inf")):
            bad = torch.where(gone[:, None], torch.full_like(x, poison), x)
            out = _run(bad, yy, w, b, 0.1)
            for k in out:
                assert torch.equal(out[k], clean[k]), (label, poison, k)
        assert not clean["row_loss"][gone].any() and not clean["grad_tokens"][gone].any()
        # ... and the others are as if they were not there
        kept = _run(x[~gone].contiguous(), y[~gone].contiguous(), w, b, 0.1)
        ref, bound = class_loss(x[~gone], y[~gone], w, b, 0.1)
        check(clean["loss"], ref["loss"], bound["loss"], "loss")
        check(clean["grad_weight"], ref["grad_weight"], bound["grad_weight"], "grad_weight")
        assert torch.equal(clean["row_loss"][~gone], kept["row_loss"])


@pytest.mark.parametrize("M", [1, 300, 5000])
def test_no_row_left(M):
    x, y, w, b = _inputs(6, M, 64, 700)
    x.fill_(float("nan"))
    out = _run(x, torch.full_like(y, -1), w, b, 0.1)
    for k, v in out.items():
        assert not torch.isnan(v).any() and not v.any(), k


def test_classes_ruled_out_by_their_bias():
    M, D, V = 300, 64, 1000
    x, y, w, b = _inputs(7, M, D, V)
    y = y % 400
    plain = _check(x, y, w[:400].contiguous(), b[:400].contiguous(), what="fewer classes")
    for low in (-float("inf"), torch.finfo(torch.float32).min):
        bias = b.clone()
        bias[400:] = low  # whole tiles of classes, and part of one
        out = _run(x, y, w, bias)
        assert not out["grad_weight"][400:].any() and not out["grad_bias"][400:].any()
        ref, bound = class_loss(x, y, w[:400], b[:400], 0.0)
        for k in ("loss", "row_loss", "grad_tokens"):
            check(out[k], ref[k], bound[k], f"{low} {k}")
        assert abs(float(out["loss"]) - float(plain["loss"])) < 1e-5


def test_values_that_are_not_finite_stay_in_their_rows():
    M, D, V = 140, 64, 700
    x, y, w, b = _inputs(8, M, D, V)
    clean = _run(x, y, w, b)
    x[9, 5] = float("nan")
    out = _run(x, y, w, b)
    rest = torch.arange(M, device="cuda") != 9
    assert torch.isnan(out["row_loss"][9]) and torch.isnan(out["loss"]).all()
    assert torch.equal(out["row_loss"][rest], clean["row_loss"][rest])
    assert torch.isnan(out["grad_tokens"][9]).all()
    assert torch.equal(out["grad_tokens"][rest], clean["grad_tokens"][rest])


@pytest.mark.parametrize("of_tokens,of_weight", [(1e30, 1e-30), (1e-36, 1e25), (2e-5, 1.0), (3e-39, 1.0), (1.0, 2e-5)])
def test_sizes_of_the_operands(of_tokens, of_weight):
    # powers of two bring both operands into the range of fp16, whatever theirs is
    x, y, w, b = _inputs(13, 150, 96, 260)
    x, w = (x.float() * of_tokens).to(BF16), (w.float() * of_weight).to(BF16)
    assert x.any() and torch.isfinite(x).all() and torch.isfinite(w).all()
    _check(x, y, w, b, 0.1, what=f"{of_tokens} {of_weight}")
    gone = y.clone()
    gone[::2] = -1  # the largest values are in rows that are left out
    big = x.clone()
    big[::2] = 3e38
    out, clean = _run(big, gone, w, b, 0.1), _run(x, gone, w, b, 0.1)
    assert all(torch.equal(out[k], clean[k]) for k in out)


@pytest.mark.parametrize("M", [1, 2, 7, 33, 63, 64, 65, 130])
@pytest.mark.parametrize("D,V", [(8, 3), (200, 1003), (1024, 20011)])
def test_the_loss_alone_of_few_rows(M, D, V):
    for bias, smoothing, left_out in ((True, 0.1, 0.4), (False, 0.0, 0.0)):
        x, y, w, b = _inputs(14, M, D, V, bias, left_out)
        ref, bound = class_loss(x, y, w, b, smoothing)
        x[(y < 0)] = float("nan")
        out = _run(x, y, w, b, smoothing, want=())
        for k, v in out.items():
            check(v, ref[k], bound[k], f"M{M} D{D} V{V} {k}")
        gone = _run(x, torch.full_like(y, V), w, b, smoothing, want=())
        assert not gone["loss"].any() and not gone["row_loss"].any()


def test_the_largest_width_and_pointers_on_their_values_boundaries():
    x, y, w, b = _inputs(15, 70, 8192, 330, True, 0.1)
    out = _check(x, y, w, b, 0.1, what="D8192")
    moved = [torch.cat([t.new_zeros(1), t])[1:] for t in (y, b)]
    assert all(t.data_ptr() % 8 for t in moved)
    again = _run(x, moved[0], w, moved[1], 0.1)
    assert all(torch.equal(out[k], again[k]) for k in out)


def test_offsets_past_32_bits():
    # more than 2^31 token values and 2^32 bytes; few classes, so that everything else stays small
    M, D, V = 600_000, 4096, 24
    g = torch.Generator(device="cuda").manual_seed(1)
    base = torch.randn(3001, D, generator=g, device="cuda").to(BF16)  # rows repeat with an odd period
    x = base.repeat(M // 3001 + 1, 1)[:M].contiguous()
    w = (torch.randn(V, D, generator=g, device="cuda") / 64).to(BF16)
    y = torch.randint(-3, V, (M,), generator=g, device="cuda", dtype=torch.int32)
    out = _run(x, y, w, None)
    n = int((y >= 0).sum())
    for rows in (slice(0, 900), slice(300_000, 300_900), slice(M - 900, M)):
        ref, bound = class_loss(x[rows], y[rows], w, None, 0.0)
        share = int((y[rows] >= 0).sum()) / n  # the reference divides by its own number of rows
        check(out["row_loss"][rows], ref["row_loss"], bound["row_loss"], "row_loss")
        check(out["grad_tokens"][rows], ref["grad_tokens"] * share, bound["grad_tokens"] * share, "grad_tokens")
    # the weight's gradient: sums over equal rows first
    l = base.double() @ w.double().T.contiguous()
    p = torch.softmax(l, 1)
    at = torch.arange(M, device="cuda") % 3001
    counts = torch.zeros(3001, V + 1, dtype=torch.float64, device="cuda")
    flat = at * (V + 1) + torch.where(y >= 0, y.long(), torch.full_like(at, V))
    counts.view(-1).index_add_(0, flat, torch.ones(M, dtype=torch.float64, device="cuda"))
    gsum = p * counts[:, :V].sum(1, keepdim=True) - counts[:, :V]
    want = gsum.T.contiguous() @ base.double() / n
    off = (out["grad_weight"].double() - want).norm() / want.norm()
    assert float(off) < 2.5 * U16  # one rounding of the result, an eighth of it for g, fp32 sums of 600,000 terms


def test_each_output_by_itself():
    x, y, w, b = _inputs(9, 333, 136, 1100, True, 0.1)
    whole = _run(x, y, w, b, 0.1)
    none = _run(x, y, w, b, 0.1, want=())
    assert torch.equal(none["loss"], whole["loss"]) and torch.equal(none["row_loss"], whole["row_loss"])
    for k in GRADS:
        part = _run(x, y, w, b, 0.1, want=(k,))
        assert torch.equal(part[k], whole[k]), k
    desc = mae.make_class_desc(x, y, w, b, smoothing=0.1)
    loss = torch.zeros(1, device="cuda")
    mae.mae_class_loss(desc, loss, workspace=_workspace(desc, False))
    assert torch.equal(loss, whole["loss"])


def test_gradient_against_differences():
    M, D, V, h = 48, 32, 90, 2.0 ** -4
    x, y, w, b = _inputs(10, M, D, V)
    x, w = ((t.float() * 8).round() / 8 for t in (x, w))  # t + h d and t - h d are bf16 numbers
    assert x.abs().max() < 8 and w.abs().max() < 8
    rng = torch.Generator(device="cuda").manual_seed(3)
    sign = lambda t: torch.where(torch.rand(t.shape, generator=rng, device="cuda") < 0.5, -1.0, 1.0)  # noqa: E731
    out = _run(x.to(BF16), y, w.to(BF16), b, 0.1)
    ref, bound = class_loss(x.to(BF16), y, w.to(BF16), b, 0.1)
    for name, at in (("grad_tokens", 0), ("grad_weight", 1), ("grad_bias", 2)):
        base = [x, w, b]
        d = sign(base[at])
        quotient = plain = noise = 0.0
        for s in (1, -1):
            moved = list(base)
            moved[at] = base[at] + s * h * d
            args = moved[0].to(BF16), y, moved[1].to(BF16), moved[2]
            quotient += s * float(_run(*args, 0.1, want=())["loss"].double()) / (2 * h)
            r, e = class_loss(*args, 0.1)
            plain += s * float(r["loss"]) / (2 * h)
            noise += float(e["loss"]) / (2 * h)
        assert abs(quotient - plain) <= noise, name
        exact = float((ref[name] * d.double()).sum())
        curve = abs(exact - plain)
        assert curve < 0.1 * float(ref[name].abs().sum()), name
        got = float((out[name].double() * d.double()).sum())
        assert abs(got - quotient) <= noise + curve + float(bound[name].sum()), name


def test_bits_are_the_same_again_and_nothing_is_written_behind_the_end():
    M, D, V = 1037, 264, 1531
    x, y, w, b = _inputs(11, M, D, V, True, 0.2)
    first = _run(x, y, w, b, 0.1)
    desc = mae.make_class_desc(x, y, w, b, smoothing=0.1)
    n = mae.mae_class_loss_workspace_bytes(desc, True)
    room = {"row_loss": torch.full((M + 40,), 5.0, device="cuda"),
            "grad_tokens": torch.full((M * D + 512,), 5.0, dtype=BF16, device="cuda"),
            "grad_weight": torch.full((V * D + 512,), 5.0, dtype=BF16, device="cuda"),
            "grad_bias": torch.full((V + 77,), 5.0, device="cuda")}
    ws = torch.full((n + 4096,), 0x3C, dtype=torch.uint8, device="cuda")
    loss = torch.zeros(1, device="cuda")
    for _ in range(3):
        mae.mae_class_loss(desc, loss, room["row_loss"], room["grad_tokens"], room["grad_weight"], room["grad_bias"],
                           ws[:n])
        assert torch.equal(loss, first["loss"])
        for k, t in room.items():
            m = first[k].numel()
            assert torch.equal(t[:m], first[k].reshape(-1)) and bool((t[m:] == 5.0).all()), k
        assert bool((ws[n:] == 0x3C).all())


def test_side_stream_replays_of_a_graph_and_new_labels():
    M, D, V = 600, 192, 1000
    x, y, w, b = _inputs(12, M, D, V)
    y2 = torch.where(torch.rand(M, device="cuda") < 0.6, torch.full_like(y, -1), y.flip(0))
    want = [_run(x, t, w, b, 0.1) for t in (y, y2)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = _run(x, y, w, b, 0.1, stream=side)
    side.synchronize()
    assert all(torch.equal(got[k], want[0][k]) for k in got)
    labels = y.clone()
    desc = mae.make_class_desc(x, labels, w, b, smoothing=0.1)
    ws = _workspace(desc, True)
    out = {k: torch.empty_like(v) for k, v in want[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mae.mae_class_loss(desc, *out.values(), ws, stream=torch.cuda.current_stream())
    for k in range(4):  # the number of rows that take part changes from replay to replay
        for t in out.values():
            t.fill_(float("nan"))
        ws.fill_(0xFF)
        labels.copy_((y, y2)[k % 2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            assert torch.equal(t, want[k % 2][name]), (k, name)


@pytest.mark.parametrize("M,D,V", [(37, 64, 1003), (600, 192, 1000), (2060, 72, 4100)])
def test_without_a_bias_the_same_bits_in_replays_of_a_graph_and_by_itself(M, D, V):
    x, y, w, _ = _inputs(19, M, D, V, False, 0.2)
    y2 = torch.where(torch.rand(M, device="cuda") < 0.5, torch.full_like(y, V), y.flip(0))
    want = [_run(x, t, w, None) for t in (y, y2)]
    none = _run(x, y, w, None, want=())
    assert all(torch.equal(none[k], want[0][k]) for k in none)
    for k in ("grad_tokens", "grad_weight"):
        assert torch.equal(_run(x, y, w, None, want=(k,))[k], want[0][k])
    labels = y.clone()
    desc = mae.make_class_desc(x, labels, w)
    n = mae.mae_class_loss_workspace_bytes(desc, True)
    ws = torch.full((n + 4096,), 0x3C, dtype=torch.uint8, device="cuda")
    out = {k: torch.empty_like(v) for k, v in want[0].items()}
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mae.mae_class_loss(desc, out["loss"], out["row_loss"], out["grad_tokens"], out["grad_weight"], None, ws[:n],
                           stream=torch.cuda.current_stream())
    for k in range(4):
        for t in out.values():
            t.fill_(float("nan"))
        ws[:n].fill_((0xFF, 0x00)[k // 2])
        labels.copy_((y, y2)[k % 2])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for name, t in out.items():
            assert torch.equal(t, want[k % 2][name]), (k, name)
        assert bool((ws[n:] == 0x3C).all())
