"""Inputs, plain forms in double precision and error bounds for the tests of the lookups and of the distillation.

Bounds: u = 2^-24 (2^-53 for float64 sums), eps/2 of the output's type per rounding.  A sum of t products in any order is off by at
most (t + 2) u sum|terms| (one rounding per product, t - 1 per addition, and the rounding of the scale; higher orders are
covered by one more u); subnormal results by half of the type's smallest subnormal.
"""
import math

import torch

DTYPES = (torch.float64, torch.float32, torch.bfloat16, torch.float16)
PADDING = (-1, -100, -2 ** 31, 2 ** 31 - 1)


def unit(dtype):
    return 2.0 ** -53 if dtype == torch.float64 else 2.0 ** -24


def half_step(dtype, value):
    """The error of one rounding of `value` to the type."""
    info = torch.finfo(dtype)
    return value.abs() * (info.eps / 2) + info.smallest_normal * info.eps / 2


def matrix(rows, cols, dtype, gen, pad=0, offset=0, spread=1.0):
    """A random matrix whose rows have a stride of cols + pad, `offset` elements into its buffer; (matrix, buffer)."""
    buffer = torch.full((offset + rows * (cols + pad),), 7.0, dtype=dtype, device="cuda")
    view = buffer[offset:].view(rows, cols + pad)[:, :cols]
    view.copy_(torch.randn((rows, cols), generator=gen, device="cuda", dtype=torch.float64) * spread)
    return view, buffer


def rows_of(rowptr, m, nnz):
    """The row of every entry, -1 for entries of no row."""
    at = torch.arange(nnz, device="cuda")
    if rowptr is None:
        return torch.div(at, max(nnz // max(m, 1), 1), rounding_mode="floor")
    row = torch.searchsorted(rowptr, at, right=True) - 1
    return torch.where((at >= rowptr[0]) & (at < rowptr[-1]), row, -1)


def dense(ids, rowptr, weights, m, n):
    """(A, |A|, entries per row, entries per column) in double precision."""
    flat = ids.reshape(-1).long()
    row = rows_of(rowptr, m, flat.numel())
    held = (flat >= 0) & (flat < n) & (row >= 0)
    w = torch.ones(flat.numel(), dtype=torch.float64, device="cuda") if weights is None else weights.reshape(-1).double()
    place = (row * n + flat)[held]
    out = []
    for values in (w[held], w[held].abs()):
        out.append(torch.zeros(m * n, dtype=torch.float64, device="cuda").index_add_(0, place, values).view(m, n))
    ones = torch.ones(int(held.sum()), dtype=torch.float64, device="cuda")
    out.append(torch.zeros(m, dtype=torch.float64, device="cuda").index_add_(0, row[held], ones))
    out.append(torch.zeros(n, dtype=torch.float64, device="cuda").index_add_(0, flat[held], ones))
    return out


def check(got, expected, bound):
    assert got.shape == expected.shape
    over = ((got.double() - expected).abs() - bound)
    assert not torch.isnan(over).any(), "NaN where there should be none, or the other way round"
    worst = over.max().item() if over.numel() else 0.0
    assert worst <= 0, f"off by {worst} more than the bound, at {int(over.argmax())}"


def check_lookup(y, ids, e, rowptr, weights, scale):
    m, n = y.shape[0], e.shape[0]
    a, size, per_row, _ = dense(ids, rowptr, weights, m, n)
    expected, magnitude = a @ e.double() * scale, size @ e.double().abs() * abs(scale)
    check(y, expected, (per_row[:, None] + 4) * unit(y.dtype) * magnitude + half_step(y.dtype, expected) * (1 + 2 ** -10))


def check_grad(de, ids, dy, rowptr, weights, scale, old=None):
    m, n = dy.shape[0], de.shape[0]
    a, size, _, per_id = dense(ids, rowptr, weights, m, n)
    expected, magnitude = a.t() @ dy.double() * scale, size.t() @ dy.double().abs() * abs(scale)
    if old is not None:
        expected, magnitude = expected + old.double(), magnitude + old.double().abs()
    check(de, expected, (per_id[:, None] + 6) * unit(dy.dtype) * magnitude + half_step(de.dtype, expected) * (1 + 2 ** -10))


def check_grad_weights(dw, ids, e, dy, rowptr, scale):
    flat, n = ids.reshape(-1).long(), e.shape[0]
    row = rows_of(rowptr, dy.shape[0], flat.numel())
    held = (flat >= 0) & (flat < n) & (row >= 0)
    x, g = e[flat.clamp(0, max(n - 1, 0))].double(), dy[row.clamp(min=0)].double()
    expected = torch.where(held, (x * g).sum(1), 0.0) * scale
    magnitude = torch.where(held, (x * g).abs().sum(1), 0.0) * abs(scale)
    check(dw.reshape(-1), expected, (e.shape[1] + 4) * unit(e.dtype) * magnitude + half_step(dw.dtype, expected))


# ------------------------------------------------------------------------------------------
# Distillation
# ------------------------------------------------------------------------------------------
def distill_plain(logits, ids, teacher, rowptr, teacher_lse, row_weights, tau, scale):
    """(loss, lse, gradient) and their error bounds before the rounding to the output's type, in double precision, row by row.

    Bounds.  An exponential of the teacher: expf is off by 2 steps of 2^-23, its argument a (|z - largest| / tau) by 2 roundings:
    d_t = 2^-22 + 2^-23 a.  One of the student: 2^-22 (ex2.approx), its argument, b in units of ln 2, by the roundings of the
    factor and of the multiply-add, 2^-23 b ln 2.  Sum of a row: every thread adds up to c = n / 512 + 16 terms and corrects its sum
    at most as often (2^-22 and 2^-23 of the exponent each, below 2^-21 as long as the exponents of corrections sum to less than 2^10),
    then 15 levels of joining: D = (2 c + 60) 2^-22 + the mean of the terms' own errors.  An exponential below 2^-126 is 0 (ex2.approx.ftz flushes what
    would be subnormal): off by up to 2^-126, times the gradient's factor where that is not in the exponent already.
    """
    m, n = logits.shape
    nnz = ids.numel()
    bounds = rowptr.tolist() if rowptr is not None else [i * (nnz // max(m, 1)) for i in range(m + 1)]
    flat, z_all = ids.reshape(-1).long(), teacher.reshape(-1).double()
    loss, lse, loss_b, lse_b = (torch.zeros(m, dtype=torch.float64, device="cuda") for _ in range(4))
    grad, grad_b = (torch.zeros((m, n), dtype=torch.float64, device="cuda") for _ in range(2))
    c = n / 512 + 16
    for i in range(m):
        at, z = flat[bounds[i]:bounds[i + 1]], z_all[bounds[i]:bounds[i + 1]] / tau
        held = (at >= 0) & (at < n) & (z != -math.inf)
        r = 1.0 if row_weights is None else float(row_weights[i])
        if r == 0.0 or not held.any():
            continue
        at, z = at[held], z[held]
        top = z.max()
        logp = z - top - ((z - top).exp().sum().log() if teacher_lse is None else float(teacher_lse[i]) - top)
        p = logp.exp()
        mass = float(p.sum())
        x = logits[i].double() / tau
        most = x.max()
        rest = (x - most).exp().sum().log()
        lse[i] = most + rest
        logq = x - most - rest
        q = logq.exp()
        terms = torch.where(p > 0, p * (logp - logq[at]), 0.0)
        loss[i] = scale * r * terms.sum()
        grad[i] = (q * mass).scatter_add(0, at, -p) * (scale * r / tau)
        # bounds
        d = 2.0 ** -22 + 2.0 ** -23 * (top - z).clamp(max=200.0)
        own = 2.0 ** -22 + 2.0 ** -23 * (-logq).clamp(max=200.0)
        total = (2 * c + 60) * 2.0 ** -22 + float((q * own).sum())
        lse_b[i] = total + 2.0 ** -40 * abs(float(lse[i]))
        spread = torch.where(p > 0, p * d * ((logp - logq[at]).abs() + 1), 0.0).sum() * 2
        loss_b[i] = abs(scale * r) * (spread + mass * (total + 2.0 ** -22)) + 2.0 ** -23 * loss[i].abs()
        pd = (p * (2 * d + 2.0 ** -22)).sum()  # the norm takes part in the errors of all
        per_id = torch.zeros(n, dtype=torch.float64, device="cuda").scatter_add(0, at, p * (d + pd / max(mass, 1e-300) + 2.0 ** -22 + at.numel() * 2.0 ** -24))
        grad_b[i] = (mass * q * (own + total + 2.0 ** -22 + 2.0 ** -23 * (1 + abs(float(lse[i]))) + pd) + per_id) * abs(scale * r / tau) + 2.0 ** -126 * (1 + mass * abs(scale * r / tau))
    return (loss, lse, grad), (loss_b, lse_b, grad_b)


def check_distill(got, logits, ids, teacher, rowptr=None, teacher_lse=None, row_weights=None, tau=1.0, scale=None):
    """got: (loss, lse, gradient); None where there is none."""
    scale = tau * tau if scale is None else scale
    expected, bounds = distill_plain(logits, ids, teacher, rowptr, teacher_lse, row_weights, tau, scale)
    for g, e, b in zip(got, expected, bounds):
        if g is not None:
            check(g, e, b + half_step(g.dtype, e) * (1 + 2 ** -10))
