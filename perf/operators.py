"""The operators at the two ends of a model over a vocabulary, as timed cases over the public entry points of the binding.

At the input end rows of ids (a CSR matrix A) meet a table E: the lookup Y = s A E, its gradient s A^T dY by sorted ids, and the
gradient of the weights.  At the output end a teacher's top logits (CSR rows of ids and logits) meet a student's dense logits: the
distillation loss of every row and its gradient.

A case is ``{"op": operator, "dtype": type of the dense matrices, sizes...}``.  ``k`` is the number of ids of a row; ``ragged``
rows have 0 to ``k`` of them and come with row pointers.  Outputs of the plain form are computed in single precision (sums over the
occurrences of an id, which may be thousands, in double) and rounded once.
"""
from __future__ import annotations

import math

import torch

own = False

_DT = {"f64": torch.float64, "f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
_SIZE = {"f64": 8, "f32": 4, "bf16": 2, "f16": 2}


def listed():
    return [
        # A decoding step: the embeddings of one token for each of 16 sequences.  Latency is all.
        {"name": "lookup_16_p1024_bf16", "op": "lookup", "dtype": "bf16", "m": 16, "k": 1, "ragged": False, "n": 1 << 15, "p": 1024, "weights": False},
        # A packed training batch with padded places.
        {"name": "lookup_20011_p4096_bf16", "op": "lookup", "dtype": "bf16", "m": 20_011, "k": 1, "ragged": False, "n": 1 << 17, "p": 4096, "weights": False},
        # Sums over weighted sets of up to 140 of 4 million features (the shape of the binary overlap workload).
        {"name": "lookup_bags_20000_d140_p64_f32", "op": "lookup", "dtype": "f32", "m": 20_000, "k": 140, "ragged": True, "n": 1 << 22, "p": 64, "weights": True},
        # Gradient of a short batch, an odd width, a dense result.
        {"name": "lookup_grad_511_p1000_f32", "op": "lookup_grad", "dtype": "f32", "gdtype": "f32", "m": 511, "k": 1, "ragged": False, "n": 1 << 15, "p": 1000, "weights": False},
        # Gradient of a training batch in half precision, kept in single precision.
        {"name": "lookup_grad_16384_p4096_bf16", "op": "lookup_grad", "dtype": "bf16", "gdtype": "f32", "m": 1 << 14, "k": 1, "ragged": False, "n": 50_021, "p": 4096, "weights": False},
        # Backward pass of small weighted sets: the table's gradient and the weights'.
        {"name": "lookup_backward_301_d20_p256_bf16", "op": "lookup_backward", "dtype": "bf16", "gdtype": "bf16", "m": 301, "k": 20, "ragged": True, "n": 60_001, "p": 256, "weights": True},
        # Backward pass of the large weighted sets.
        {"name": "lookup_backward_20000_d140_p64_f32", "op": "lookup_backward", "dtype": "f32", "gdtype": "f32", "m": 20_000, "k": 140, "ragged": True, "n": 1 << 22, "p": 64, "weights": True},
        # A few positions of a small vocabulary, loss and gradient at once.  Latency is all.
        {"name": "distill_step_17_n32768_k16_f32", "op": "distill_step", "dtype": "f32", "t": 17, "n": 1 << 15, "ld": 1 << 15, "k": 16, "ragged": False, "temperature": 1.0, "left_out": 0.0},
        # Few positions over a large vocabulary, the loss and later its gradient.
        {"name": "distill_pair_9_n131072_k500_bf16", "op": "distill_pair", "dtype": "bf16", "t": 9, "n": 1 << 17, "ld": 1 << 17, "k": 500, "ragged": False, "temperature": 2.0, "left_out": 0.0},
        # An odd vocabulary in rows of an odd stride, ragged teacher rows, a quarter of the positions (prompts) left out.
        {"name": "distill_pair_1999_n50021_k64_f16", "op": "distill_pair", "dtype": "f16", "t": 1999, "n": 50_021, "ld": 50_023, "k": 64, "ragged": True, "temperature": 1.0, "left_out": 0.25},
        # Loss and gradient at once, single precision.
        {"name": "distill_step_255_n100003_k200_f32", "op": "distill_step", "dtype": "f32", "t": 255, "n": 100_003, "ld": 100_004, "k": 200, "ragged": True, "temperature": 1.5, "left_out": 0.0},
        # Loss and gradient of a training batch at once.
        {"name": "distill_step_4096_n131072_k64_bf16", "op": "distill_step", "dtype": "bf16", "t": 4096, "n": 1 << 17, "ld": 1 << 17, "k": 64, "ragged": False, "temperature": 1.0, "left_out": 0.0},
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the operators, types and size ranges that the listed cases stand for."""
    op = rng.choice(("lookup", "lookup", "lookup_grad", "lookup_backward", "distill_pair", "distill_step", "distill_step"))
    if op.startswith("lookup"):
        bags = op == "lookup_backward" or rng.random() < 0.4
        dtype = rng.choice(("bf16", "f16", "f32", "f32", "f64"))
        p = _log_int(rng, 16, 1024 if bags else 6000)
        if rng.random() < 0.6:
            p = (p + 7) // 8 * 8
        n = _log_int(rng, 500, min(1 << 21, (1 << 28) // p))
        k = _log_int(rng, 2, 150) if bags else 1
        m = _log_int(rng, 1, max(1, min(30_000, (1 << 27) // (p * k))))
        case = {"op": op, "dtype": dtype, "m": m, "k": k, "ragged": bags and rng.random() < 0.7, "n": n, "p": p,
                "weights": bags and (op == "lookup_backward" or rng.random() < 0.5)}
        if op != "lookup":
            case["gdtype"] = dtype if dtype in ("f32", "f64") else rng.choice((dtype, "f32"))
        return case
    n = _log_int(rng, 1000, 200_000)
    t = _log_int(rng, 1, max(1, min(4096, (1 << 28) // n)))
    return {"op": op, "dtype": rng.choice(("bf16", "bf16", "f16", "f32")), "t": t, "n": n, "ld": n + rng.choice((0, 0, 1, 8, 37)), "k": min(_log_int(rng, 4, 700), n // 2),
            "ragged": rng.random() < 0.5, "temperature": rng.choice((1.0, 1.5, 2.0, 4.0)), "left_out": rng.choice((0.0, 0.0, 0.3))}


# ------------------------------------------------------------------------------------------
# Inputs
# ------------------------------------------------------------------------------------------
def _zipf(shape, n, gen):
    """Ids of a bounded Zipf distribution (exponent 1.1) over a random order of the vocabulary."""
    u = torch.rand(shape, generator=gen, device="cuda", dtype=torch.float64)
    rank = ((n ** -0.1 - 1.0) * u + 1.0) ** -10.0
    order = torch.randperm(n, generator=gen, device="cuda")
    return order[(rank.long() - 1).clamp_(0, n - 1)].to(torch.int32)


def _ragged(m, k, gen):
    """Row pointers of m rows of 0 to k entries; a twentieth of the rows has none.  The lengths are the same for every seed,
    their order is not."""
    at = torch.arange(m, device="cuda")
    length = torch.where(at % 20 == 19, 0, k // 3 + 1 + at * 7919 % (k - k // 3))[torch.randperm(m, generator=gen, device="cuda")]
    rowptr = torch.zeros(m + 1, dtype=torch.int64, device="cuda")
    torch.cumsum(length, 0, out=rowptr[1:])
    return rowptr


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    dt = _DT[case["dtype"]]
    s = {"case": case}
    if case["op"].startswith("lookup"):
        m, k, n, p = case["m"], case["k"], case["n"], case["p"]
        s["rowptr"] = _ragged(m, k, gen) if case["ragged"] else None
        nnz = int(s["rowptr"][-1]) if case["ragged"] else m * k
        ids = _zipf((nnz,), n, gen)
        ids[torch.rand(nnz, generator=gen, device="cuda") < 0.03] = -1  # padded places
        s["ids"] = ids if case["ragged"] or k == 1 else ids.view(m, k)
        wdt = torch.float64 if dt == torch.float64 else torch.float32
        s["weights"] = torch.rand(s["ids"].shape, generator=gen, device="cuda", dtype=wdt) + 0.5 if case["weights"] else None
        s["scale"] = math.sqrt(p)
        if case["op"] != "lookup_grad":
            s["e"] = torch.randn((n, p), generator=gen, device="cuda", dtype=dt).mul_(0.02)
        if case["op"] != "lookup":
            s["dy"] = torch.randn((m, p), generator=gen, device="cuda", dtype=dt)
        return s
    t, n, k = case["t"], case["n"], case["k"]
    s["rowptr"] = _ragged(t, k, gen) if case["ragged"] else None
    logits = torch.randn((t, case["ld"]), generator=gen, device="cuda", dtype=dt).mul_(2.0)[:, :n]
    # k distinct ids a row in the order of the teacher's logits, which fall; the student has an idea of them
    place = torch.rand((t, k), generator=gen, device="cuda", dtype=torch.float64)
    ids = ((torch.arange(k, device="cuda") + place) * (n / k)).long().clamp_(0, n - 1)
    ids = ids.gather(1, torch.rand((t, k), generator=gen, device="cuda").argsort(1))
    falling = 14.0 - 2.0 * torch.log1p(torch.arange(k, device="cuda", dtype=torch.float32))
    teacher = falling + 0.3 * torch.randn((t, k), generator=gen, device="cuda")
    logits.scatter_add_(1, ids, (0.8 * teacher).clamp_(min=0.0).to(dt))
    if case["ragged"]:
        kept = torch.arange(k, device="cuda") < (s["rowptr"][1:] - s["rowptr"][:-1])[:, None]
        ids, teacher = ids[kept], teacher[kept]
    s["logits"], s["ids"], s["teacher"] = logits, ids.to(torch.int32).contiguous(), teacher.to(dt).contiguous()
    s["row_weights"] = None
    if case["left_out"]:
        # the mean over the positions, times the loss scale that half precision gradients are trained with
        s["row_weights"] = (torch.rand(t, generator=gen, device="cuda") >= case["left_out"]).float() * ((65536.0 if dt == torch.float16 else 1.0) / t)
    return s


# ------------------------------------------------------------------------------------------
# One pass
# ------------------------------------------------------------------------------------------
def _rows_of(s, m):
    """The row of every entry."""
    if s["rowptr"] is None:
        return torch.arange(m, device="cuda").repeat_interleave(s["ids"].numel() // m)
    return torch.repeat_interleave(torch.arange(m, device="cuda"), s["rowptr"][1:] - s["rowptr"][:-1], output_size=s["ids"].numel())


def _plain_lookup(s):
    case, e = s["case"], s["e"]
    wide = torch.float64 if e.dtype == torch.float64 else torch.float32
    ids = s["ids"].reshape(-1).long()
    held = ids >= 0
    x = e[ids.clamp(min=0)].to(wide)
    w = held.to(wide) * s["scale"]
    if s["weights"] is not None:
        w = w * s["weights"].reshape(-1)
    x *= w[:, None]
    if case["ragged"]:
        x = torch.zeros((case["m"], case["p"]), dtype=wide, device="cuda").index_add_(0, _rows_of(s, case["m"]), x)
    elif case["k"] > 1:
        x = x.view(case["m"], case["k"], case["p"]).sum(1)
    return x.to(e.dtype)


def _plain_lookup_grad(s):
    case, dy = s["case"], s["dy"]
    ids = s["ids"].reshape(-1).long()
    held = ids >= 0
    x = dy.double() if case["k"] == 1 and not case["ragged"] else dy.double()[_rows_of(s, case["m"])]
    w = held.double() * s["scale"]
    if s["weights"] is not None:
        w = w * s["weights"].reshape(-1)
    sums = torch.zeros((case["n"], case["p"]), dtype=torch.float64, device="cuda")
    return sums.index_add_(0, ids.clamp(min=0), x * w[:, None]).to(_DT[case["gdtype"]])


def _plain_lookup_grad_weights(s):
    case, e = s["case"], s["e"]
    wide = torch.float64 if e.dtype == torch.float64 else torch.float32
    ids = s["ids"].reshape(-1).long()
    dots = (e[ids.clamp(min=0)].to(wide) * s["dy"].to(wide)[_rows_of(s, case["m"])]).sum(1)
    return (torch.where(ids >= 0, dots, 0.0) * s["scale"]).view(s["ids"].shape)


def _plain_distill(s, lse_kept=None, grad=True):
    """(loss, lse, gradient), or the gradient from a kept lse."""
    case = s["case"]
    t, tau = case["t"], case["temperature"]
    scale = tau * tau
    rows, ids = _rows_of(s, t), s["ids"].reshape(-1).long()
    x = s["logits"].float() / tau
    w = torch.ones(t, device="cuda") if s["row_weights"] is None else s["row_weights"]
    z = s["teacher"].reshape(-1).float() / tau
    top = torch.full((t,), -math.inf, device="cuda").index_reduce_(0, rows, z, "amax")
    held = (torch.bincount(rows, minlength=t) > 0) & (w != 0)
    ez = torch.exp(z - top[rows])
    total = torch.zeros(t, device="cuda").index_add_(0, rows, ez)
    logp = z - (top + torch.log(total))[rows]
    pt = torch.exp(logp)
    if lse_kept is None:
        most = x.amax(1)
        lse = most + torch.log(torch.exp(x - most[:, None]).sum(1))
    else:
        lse = lse_kept
    out = []
    if lse_kept is None:
        terms = pt * (logp - (x[rows, ids] - lse[rows]))
        loss = scale * w * torch.zeros(t, device="cuda").index_add_(0, rows, terms)
        out += [torch.where(held, loss, 0.0), torch.where(held, lse, 0.0)]
    if grad:
        g = torch.exp(x - lse[:, None])
        g.index_put_((rows, ids), -pt, accumulate=True)
        g *= (torch.where(held, w, 0.0) * (scale / tau))[:, None]
        out.append(g.to(s["logits"].dtype))
    return out


def run(state):
    s, op = state, state["case"]["op"]
    if not own:
        if op == "lookup":
            return _plain_lookup(s)
        if op == "lookup_grad":
            return _plain_lookup_grad(s)
        if op == "lookup_backward":
            return [_plain_lookup_grad(s), _plain_lookup_grad_weights(s)]
        if op == "distill_pair":
            loss, lse = _plain_distill(s, grad=False)
            return [loss, lse] + _plain_distill(s, lse_kept=lse)
        return _plain_distill(s)
    from paper_2608_09713_b200 import binding as B
    if op == "lookup":
        return B.spsyrk_lookup(s["ids"], s["e"], rowptr=s["rowptr"], weights=s["weights"], scale=s["scale"])
    if op.startswith("lookup"):
        case = s["case"]
        de = B.spsyrk_lookup_grad(s["ids"], s["dy"], case["n"], rowptr=s["rowptr"], weights=s["weights"], scale=s["scale"], dtype=_DT[case["gdtype"]])
        if op == "lookup_grad":
            return de
        return [de, B.spsyrk_lookup_grad_weights(s["ids"], s["e"], s["dy"], rowptr=s["rowptr"], scale=s["scale"])]
    teacher = dict(rowptr=s["rowptr"], row_weights=s["row_weights"], temperature=s["case"]["temperature"])
    if op == "distill_pair":
        loss, lse = B.spsyrk_distill(s["logits"], s["ids"], s["teacher"], **teacher)
        return [loss, lse, B.spsyrk_distill_grad(s["logits"], lse, s["ids"], s["teacher"], **teacher)]
    return list(B.spsyrk_distill(s["logits"], s["ids"], s["teacher"], grad=True, **teacher))


# ------------------------------------------------------------------------------------------
# What a pass cannot do without
# ------------------------------------------------------------------------------------------
def _distinct(n, draws):
    """Ids that `draws` draws of the Zipf distribution are expected to hold, by pieces of its inverse."""
    steps = 4096
    c = 1.0 - n ** -0.1
    total, lo = 0.0, 1.0
    for i in range(1, steps + 1):
        hi = (n + 1.0) ** (i / steps)
        share = max((min(lo, n) ** -0.1 - min(hi, n) ** -0.1) / c, 0.0) / max(hi - lo, 1e-9)
        total += (hi - lo) * -math.expm1(draws * math.log1p(-min(share, 0.999999)))
        lo = hi
    return min(total, n, draws)


def work(case):
    if case["op"].startswith("lookup"):
        m, n, p, sv = case["m"], case["n"], case["p"], _SIZE[case["dtype"]]
        nnz = m * case["k"] if not case["ragged"] else 0.95 * m * (2 * case["k"] / 3 + 0.5)
        sw = (8 if case["dtype"] == "f64" else 4)
        index = nnz * 4 + (8 * (m + 1) if case["ragged"] else 0)
        table = _distinct(n, 0.97 * nnz) * p * sv
        forward = index + (nnz * sw if case["weights"] else 0) + m * p * sv
        if case["op"] == "lookup":
            return {"bytes": forward + table, "flops": 2 * nnz * p}
        back = forward + n * p * _SIZE[case["gdtype"]]  # dy is as large as y
        if case["op"] == "lookup_grad":
            return {"bytes": back, "flops": 2 * nnz * p}
        return {"bytes": back + table + nnz * sw, "flops": 4 * nnz * p}
    t, n, sv = case["t"], case["n"], _SIZE[case["dtype"]]
    entries = t * case["k"] * (1.0 if not case["ragged"] else 0.64)
    live = t * (1.0 - case["left_out"])
    read, small = live * n * sv, entries * (4 + sv) + 8 * t
    if case["op"] == "distill_step":
        return {"bytes": read + small + t * n * sv, "flops": 8 * live * n}
    return {"bytes": 2 * (read + small) + t * n * sv, "flops": 8 * live * n}


# ------------------------------------------------------------------------------------------
# The definition in double precision
# ------------------------------------------------------------------------------------------
def _csr(s, m, n, values):
    """The matrix A of a lookup in double precision, padded places left out, entries of the same place added up."""
    ids = s["ids"].reshape(-1)
    if s["rowptr"] is None:
        row = torch.div(torch.arange(ids.numel(), device="cuda"), s["case"]["k"], rounding_mode="floor")
    else:
        row = torch.searchsorted(s["rowptr"], torch.arange(ids.numel(), device="cuda"), right=True) - 1
    held = ids >= 0
    return torch.sparse_coo_tensor(torch.stack((row[held], ids[held].long())), values[held], (m, n)).coalesce()


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"].startswith("lookup"):
        m, n = case["m"], case["n"]
        ones = torch.ones(s["ids"].numel(), dtype=torch.float64, device="cuda")
        a = _csr(s, m, n, ones if s["weights"] is None else s["weights"].reshape(-1).double())
        if case["op"] == "lookup":
            return torch.sparse.mm(a, s["e"].double()) * s["scale"]
        de = torch.sparse.mm(a.t().coalesce(), s["dy"].double()) * s["scale"]
        if case["op"] == "lookup_grad":
            return de
        dw = torch.zeros(s["ids"].numel(), dtype=torch.float64, device="cuda")
        ids = s["ids"].reshape(-1)
        for begin in range(0, ids.numel(), 1 << 18):  # a piece of the entries at a time
            at = torch.arange(begin, min(begin + (1 << 18), ids.numel()), device="cuda")
            row = torch.div(at, case["k"], rounding_mode="floor") if s["rowptr"] is None else torch.searchsorted(s["rowptr"], at, right=True) - 1
            inside = ids[at] >= 0
            pair = torch.einsum("tp,tp->t", s["e"][ids[at][inside].long()].double(), s["dy"][row[inside]].double())
            dw[at[inside]] = pair * s["scale"]
        return [de, dw.view(s["ids"].shape)]
    t, n, tau = case["t"], case["n"], case["temperature"]
    loss, lse = (torch.zeros(t, dtype=torch.float64, device="cuda") for _ in range(2))
    grad = torch.zeros((t, n), dtype=torch.float64, device="cuda")
    bounds = [i * case["k"] for i in range(t + 1)] if s["rowptr"] is None else s["rowptr"].tolist()
    flat_ids, flat_z = s["ids"].reshape(-1).long(), s["teacher"].reshape(-1).double()
    weights = [1.0] * t if s["row_weights"] is None else s["row_weights"].double().tolist()
    for i in range(t):  # row by row, as the definition stands
        b, e = bounds[i], bounds[i + 1]
        if b == e or weights[i] == 0.0:
            continue
        z, x = flat_z[b:e] / tau, s["logits"][i].double() / tau
        log_p = z - torch.logsumexp(z, 0)
        norm = torch.logsumexp(x, 0)
        log_q = x - norm
        lse[i] = norm
        loss[i] = tau * tau * weights[i] * torch.dot(log_p.exp(), log_p - log_q[flat_ids[b:e]])
        g = log_q.exp()
        g.scatter_add_(0, flat_ids[b:e], -log_p.exp())
        grad[i] = g * (tau * weights[i])
    return [loss, lse, grad]
