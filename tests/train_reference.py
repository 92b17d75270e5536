"""Plain 64-bit forms of the operators around the encoder, and bounds of what fp32 arithmetic may lose in
them.  U32, U16: the largest relative error of one rounding to fp32 / bf16 (half of finfo.eps)."""
from __future__ import annotations

import numpy as np
import torch

U32 = torch.finfo(torch.float32).eps / 2
U16 = torch.finfo(torch.bfloat16).eps / 2
TINY = 6e-41  # half a step of the smallest bf16 numbers, and above 0

MASK64 = (1 << 64) - 1
GAMMA = 0x9E3779B97F4A7C15


def rounding(dtype):
    return U16 if dtype == torch.bfloat16 else U32


def check(got, want, bound, what):
    """|got - want| <= bound, element by element, in 64 bits on the tensors' device; NaN fails."""
    got = got.double().reshape(want.shape)
    err = (got - want).abs()
    bad = ~(err <= bound + TINY)
    if bool(bad.any()):
        score = torch.where(torch.isnan(err), torch.full_like(err, float("inf")), err / (bound + TINY))
        i = int(score.argmax().item())
        limit = torch.as_tensor(bound, dtype=torch.float64).expand_as(err).flatten()[i].item()
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values out of bounds; worst at {i}: got "
                             f"{got.flatten()[i].item()!r}, want {want.flatten()[i].item()!r}, bound {limit:.3e}")


# ---- layer norm ------------------------------------------------------------------------------------
# A row's sums are made of sums over lanes (at most 8 groups of 4 values each), 6 exchanges between lanes
# and 2 additions of wavefronts: no value passes more than DEPTH additions.
DEPTH = 20


def layer_norm(x, weight, bias, eps):
    """-> y, mean, rstd and the bounds of their fp32 errors (before y is rounded to its type)."""
    x = x.double()
    w = torch.ones_like(x[0]) if weight is None else weight.double()
    b = torch.zeros_like(x[0]) if bias is None else bias.double()
    mean = x.mean(1)
    d = x - mean[:, None]
    var = d.square().mean(1)
    rstd = 1.0 / torch.sqrt(var + eps)
    h = d * rstd[:, None]
    y = h * w + b
    e_mean = (DEPTH + 2) * U32 * x.abs().mean(1)
    e_d = e_mean[:, None] + U32 * d.abs()
    e_var = 2 * (e_d * d.abs()).mean(1) + e_d.square().mean(1) + (DEPTH + 3) * U32 * var
    r_rstd = e_var / (2 * (var + eps)).clamp(min=TINY) + 4 * U32
    e_y = (w.abs() * (e_d * rstd[:, None] + h.abs() * (r_rstd[:, None] + 3 * U32))) * 1.01 + U32 * (y.abs() + b.abs())
    return (y, mean, rstd), (e_y, e_mean, r_rstd * rstd)


def layer_norm_grad(x, grad_y, weight, mean, rstd, rows_in_turn):
    """rows_in_turn: rows that one lane adds up one after the other."""
    x, gy = x.double(), grad_y.double()
    w = torch.ones_like(x[0]) if weight is None else weight.double()
    mean, rstd = mean.double()[:, None], rstd.double()[:, None]
    h = (x - mean) * rstd
    g = gy * w
    mg = g.mean(1, keepdim=True)
    mgh = (g * h).mean(1, keepdim=True)
    gx = (g - mg - h * mgh) * rstd
    e_gx = rstd * (4 * U32 * g.abs() + (DEPTH + 6) * U32 * g.abs().mean(1, keepdim=True)
                   + h.abs() * (DEPTH + 10) * U32 * (g * h).abs().mean(1, keepdim=True))
    gw, gb = (gy * h).sum(0), gy.sum(0)
    n = (rows_in_turn + 12) * U32
    return (gx, gw, gb), (e_gx, n * (gy * h).abs().sum(0), n * gy.abs().sum(0))


# ---- dropout -----------------------------------------------------------------------------------------
def mix64(z):
    z &= MASK64
    z = ((z ^ (z >> 30)) * 0xBF58476D1CE4E5B9) & MASK64
    z = ((z ^ (z >> 27)) * 0x94D049BB133111EB) & MASK64
    return z ^ (z >> 31)


def dropout_key(seed, batch_index, layer):
    key = mix64(mix64(seed + GAMMA) + GAMMA * (batch_index + 1))
    return mix64(key + GAMMA * (((layer << 32) | (11 << 24)) + 1))


def dropout_keep(M, D, p, rows_per_draw, seed, batch_index, layer, row_base):
    """[M, D] of truth values: which values are kept (Python's integers for the key, NumPy's for the draws)."""
    rows = np.arange(M, dtype=np.uint64) + np.uint64(row_base)
    if rows_per_draw:
        index = np.broadcast_to((rows // np.uint64(rows_per_draw))[:, None], (M, D))
    else:
        index = rows[:, None] * np.uint64(D) + np.arange(D, dtype=np.uint64)
    z = (index >> np.uint64(1)) + np.uint64(1)
    z = np.uint64(dropout_key(seed, batch_index, layer)) + z * np.uint64(GAMMA)
    z = (z ^ (z >> np.uint64(30))) * np.uint64(0xBF58476D1CE4E5B9)
    z = (z ^ (z >> np.uint64(27))) * np.uint64(0x94D049BB133111EB)
    z = z ^ (z >> np.uint64(31))
    bits = np.where(index & np.uint64(1), z >> np.uint64(32), z & np.uint64(0xFFFFFFFF))
    return bits >= np.uint64(int(np.floor(float(np.float32(p)) * 2.0 ** 32 + 0.5)))


# ---- softmax cross entropy of a linear head --------------------------------------------------------------
def class_loss(tokens, labels, weight, bias, smoothing, grad_scale=1.0):
    """-> dict of results, dict of bounds.  The gradients' bounds are those of the stated method: logits summed in
    fp32, 2^15 g rounded to fp16 for the products; without bias and smoothing g is
    made of exponentials that were rounded so once before (those of the first piece of the classes), but for the label's."""
    dev = tokens.device
    V, D = weight.shape
    M = tokens.shape[0]
    ok = (labels >= 0) & (labels < V)
    n = int(ok.sum())
    out = {"row_loss": torch.zeros(M, dtype=torch.float64, device=dev),
           "grad_tokens": torch.zeros(M, D, dtype=torch.float64, device=dev),
           "grad_weight": torch.zeros(V, D, dtype=torch.float64, device=dev),
           "grad_bias": torch.zeros(V, dtype=torch.float64, device=dev)}
    bound = {k: torch.zeros_like(v) for k, v in out.items()}
    out["loss"] = torch.zeros(1, dtype=torch.float64, device=dev)
    bound["loss"] = torch.zeros(1, dtype=torch.float64, device=dev)
    if n == 0:
        return out, bound
    at = torch.nonzero(ok).reshape(-1)
    x, y, w = tokens[at].double(), labels[at].long(), weight.double()
    b = torch.zeros(V, dtype=torch.float64, device=dev) if bias is None else bias.double()
    r = torch.arange(n, device=dev)
    l = x @ w.T.contiguous() + b
    size = x.abs() @ w.abs().T.contiguous() + torch.where(torch.isinf(b), torch.zeros_like(b), b.abs())
    e_l = (D + 3) * U32 * size  # of a logit
    top = l.max(1, keepdim=True).values
    ex = torch.exp(l - top)
    p = ex / ex.sum(1, keepdim=True)
    lse = (top + torch.log(ex.sum(1, keepdim=True)))[:, 0]
    mean_l = l.mean(1) if smoothing else torch.zeros(n, dtype=torch.float64, device=dev)
    row = lse - (1 - smoothing) * l[r, y] - smoothing * mean_l
    # exponentials: their argument's roundings (times its size, at most 104 before the result vanishes) and the
    # function's own error, then sums of V of them over lanes, wavefronts and tiles
    rel = ((top - l).clamp(max=104.0) * ex).sum(1) / ex.sum(1) * 4 * U32 + (V + 16) * U32
    worst = e_l.max(1).values
    out["row_loss"][at] = row
    e_row = 2 * worst + rel + 4 * U32 * (lse.abs() + l[r, y].abs())
    if smoothing:
        e_row = e_row + smoothing * (V + 4) * U32 * l.abs().mean(1)
    bound["row_loss"][at] = e_row
    out["loss"] = row.sum().reshape(1) / n
    bound["loss"] = e_row.mean().reshape(1) + U32 * out["loss"].abs()
    want = torch.full_like(p, smoothing / V)
    want[r, y] += 1 - smoothing
    g = p - want
    e_g = p * (2 * worst[:, None] + rel[:, None] + 4 * U32 * (top - l).clamp(max=104.0) + 8 * U32) + 2 * U32 * (p + want)
    f = abs(grad_scale) / n
    e_round = 2.0 ** -11 * g.abs() + 2.0 ** -40  # half a step of fp16, and of its smallest numbers
    if bias is None and not smoothing:
        # an exponential under a maximum above it, e = 2^15 exp: half a step is 2^-11 of it, or 2^-40 of 1; then it is
        # multiplied by a factor of at most 1 that makes it p
        once = 2.0 ** -11 * p + 2.0 ** -40
        once[r, y] = 0.0
        e_round = e_round + once
    e_products = (V + 8) * U32 * (g.abs() @ w.abs())
    out["grad_tokens"][at] = grad_scale / n * (g @ w)
    bound["grad_tokens"][at] = f * ((e_g + e_round) @ w.abs() + e_products) + (U16 + 4 * U32) * out["grad_tokens"][at].abs()
    out["grad_weight"] = grad_scale / n * (g.T.contiguous() @ x)
    bound["grad_weight"] = (f * ((e_g + e_round).T.contiguous() @ x.abs() + (n + 8) * U32 * (g.abs().T.contiguous() @ x.abs()))
                            + (U16 + 4 * U32) * out["grad_weight"].abs())
    out["grad_bias"] = grad_scale / n * g.sum(0)
    bound["grad_bias"] = f * (e_g.sum(0) + (n + 4) * U32 * g.abs().sum(0)) + 4 * U32 * out["grad_bias"].abs()
    return out, bound
