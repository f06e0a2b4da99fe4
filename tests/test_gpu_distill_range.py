"""Distillation over all the logits and temperatures that it accepts: rows far from zero, rows masked throughout with a large number, small
and large temperatures.

Softmax is the same for a shifted row, so the bounds are those of vocabulary.distill_plain for rows shifted to a largest logit of
zero.  They count two roundings of an exponent (the factor's and the multiply-add's); a difference that is multiplied has three: 1.5 of them.
"""
import math

import pytest
import torch

import vocabulary as V

pytestmark = pytest.mark.gpu
LOGITS = (torch.float32, torch.bfloat16, torch.float16)


@pytest.fixture(scope="module")
def B():
    from paper_2608_09713_b200 import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _expected(logits, ids, z, tau, scale, teacher_lse=None):
    """(loss, lse, gradient) in double precision, their bounds, and the size of the gradient's part that is the student's."""
    expected, _ = V.distill_plain(logits, ids, z, None, teacher_lse, None, tau, scale)
    held = (ids >= 0) & (ids < logits.shape[1])
    top = torch.where(held, z.double(), -math.inf).amax(1, keepdim=True)
    s = logits.double()
    lse = None if teacher_lse is None else teacher_lse.double() - top[:, 0] / tau
    shifted, bounds = V.distill_plain(s - s.amax(1, keepdim=True), ids, z.double() - top, None, lse, None, tau, scale)
    bounds = [1.5 * b for b in bounds]
    bounds[1] = bounds[1] + 2.0 ** -40 * expected[1].abs()
    mass = 1.0 if lse is None else (torch.where(held, z.double() - top, -math.inf) / tau - lse[:, None]).exp().sum(1, keepdim=True)
    return expected, bounds, torch.softmax(s / tau, 1) * mass * abs(scale / tau)


def _check(got, expected, bound):
    V.check(got, expected, bound + V.half_step(got.dtype, expected) * (1 + 2 ** -10))


def _rows(base, dtype, n, k, spread=2.0, seed=0):
    """Every kind of student's row with every kind of teacher's: constant, spread around the base, a third far below the base, half -infinity."""
    gen = _gen(seed + n)
    below = 1.5 * base if base < 0 else base / 1.5
    ids = torch.randint(0, n // 2, (16, k), generator=gen, device="cuda", dtype=torch.int32)
    ids[:, k // 2] = -1

    def kinds(width):
        x = torch.full((4, width), float(base), device="cuda", dtype=torch.float64)
        x[1] += spread * torch.randn(width, generator=gen, device="cuda", dtype=torch.float64)
        x[2, ::3] = below
        most = torch.finfo(dtype).max / 2
        x = x.clamp(-most, most)
        x[3, width // 2:] = -math.inf
        return x.to(dtype)

    return kinds(n).repeat(4, 1), ids, kinds(k).repeat_interleave(4, 0)


# (the type's largest numbers, the numbers that masks are made of, logits at which a kernel may go over to another form)
BASES = (0.0, 300.0, 360.0, -2839.0, 2839.0, 2850.0, 5e4, -1e5, -1e9, 1e9, -1e10, 1e10, -1e12, 1e15, -1e20, 1e20, -1e29, 2e30, -3e33)
SIZES = [(333, 5), (40_001, 6), (5000, 1100)]


def _fits(base, dtype):
    return abs(base) * 1.5 < torch.finfo(dtype).max


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", LOGITS)
@pytest.mark.parametrize("base", BASES)
def test_loss_of_rows_far_from_zero(B, base, dtype, n, k):
    if not _fits(base, dtype):
        base = math.copysign(4e4, base)
    logits, ids, z = _rows(base, dtype, n, k)
    expected, bounds, student = _expected(logits, ids, z, 1.0, 1.0)
    loss, lse = B.spsyrk_distill(logits, ids, z)
    _check(loss, expected[0], bounds[0])
    _check(lse, expected[1], bounds[1])
    loss, lse, grad = B.spsyrk_distill(logits, ids, z, grad=True)
    _check(loss, expected[0], bounds[0])
    _check(lse, expected[1], bounds[1])
    if dtype == torch.float32:
        _check(grad, expected[2], bounds[2])
        B.spsyrk_distill(logits, ids, z, grad=logits)
        assert torch.equal(logits, grad)


# temperature, logits around which number, spread how far
TEMPERATURES = [(1e-6, 0.0, 3e-6), (1e-6, 10.0, 2e-6), (1e-6, 2000.0, 1e-3), (1e-6, -1e4, 1.0), (1e-3, 1.0, 2e-3), (1e-3, 20.0, 3.0), (0.01, 30.0, 0.05), (0.02, 0.0, 3.0),
                (1e3, -1e3, 3e3), (1e6, 1e3, 2e4)]


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", LOGITS)
@pytest.mark.parametrize("tau,base,spread", TEMPERATURES)
def test_loss_at_temperatures(B, tau, base, spread, dtype, n, k):
    logits, ids, z = _rows(base, dtype, n, k, spread)
    expected, bounds, student = _expected(logits, ids, z, tau, tau)
    loss, lse, grad = B.spsyrk_distill(logits, ids, z, temperature=tau, scale=tau, grad=True)
    _check(loss, expected[0], bounds[0])
    _check(lse, expected[1], bounds[1])
    if dtype == torch.float32:
        _check(grad, expected[2], bounds[2])


@pytest.mark.parametrize("base", [300.0, 2839.0, 2850.0, -2839.0, 5e4])
def test_a_given_norm_far_from_zero(B, base):
    logits, ids, z = _rows(base, torch.float32, 3000, 20)
    z[3::4] = base  # (no -infinity: a norm for every row)
    lse = z.float().amax(1) + torch.rand(16, generator=_gen(1), device="cuda") + 1.0
    expected, bounds, student = _expected(logits, ids, z, 1.0, 1.0, lse)
    loss, norm, grad = B.spsyrk_distill(logits, ids, z, teacher_lse=lse, grad=True)
    for got, e, b in zip((loss, norm, grad), expected, bounds):
        _check(got, e, b)


# Where the gradient's factor goes into the exponent, the sum of the two is rounded once more: exponents below 2^9, half a step 2^-16, of the
# student's part.
@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("base", BASES)
def test_half_precision_gradient_of_rows_far_from_zero(B, base, dtype, n, k):
    if not _fits(base, dtype):
        base = math.copysign(4e4, base)
    logits, ids, z = _rows(base, dtype, n, k)
    expected, bounds, student = _expected(logits, ids, z, 1.0, 1.0)
    grad = B.spsyrk_distill(logits, ids, z, grad=True)[2]
    _check(grad, expected[2], bounds[2] + 2.0 ** -16 * student)
    B.spsyrk_distill(logits, ids, z, grad=logits)
    assert torch.equal(logits, grad)


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float16))
@pytest.mark.parametrize("tau,base,spread", TEMPERATURES)
def test_half_precision_gradient_at_temperatures(B, tau, base, spread, dtype, n, k):
    logits, ids, z = _rows(base, dtype, n, k, spread)
    expected, bounds, student = _expected(logits, ids, z, tau, tau)
    grad = B.spsyrk_distill(logits, ids, z, temperature=tau, scale=tau, grad=True)[2]
    _check(grad, expected[2], bounds[2] + 2.0 ** -16 * student)


def test_half_precision_gradient_between_other_boundaries(B):
    """A gradient whose rows lie otherwise than the logits goes element by element."""
    for base in (2839.0, 4e4):
        logits, ids, z = _rows(base, torch.float16, 333, 5)
        expected, bounds, student = _expected(logits, ids, z, 1.0, 1.0)
        room = torch.zeros(16 * 335 + 3, dtype=torch.float16, device="cuda")
        grad = B.spsyrk_distill(logits, ids, z, grad=room[3:].view(16, 335)[:, :333])[2]
        _check(grad, expected[2], bounds[2] + 2.0 ** -16 * student)


# The gradient from a kept lse: a float below 2^10 is off by 2^-24 of itself; of a larger one nothing is asked.
def _check_kept(B, logits, ids, z, tau):
    expected, bounds, student = _expected(logits, ids, z, tau, tau)
    bound = bounds[2] + (2.0 ** -16 + 2.0 ** -24 * expected[1].abs().clamp(max=1024.0)[:, None]) * student
    lse = B.spsyrk_distill(logits, ids, z, temperature=tau, scale=tau)[1]
    grad = B.spsyrk_distill_grad(logits, lse, ids, z, temperature=tau, scale=tau)
    _check(grad, expected[2], bound)
    B.spsyrk_distill_grad(logits, lse, ids, z, temperature=tau, scale=tau, grad=logits)
    assert torch.equal(logits, grad)


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", LOGITS)
@pytest.mark.parametrize("base", BASES + (1000.0, 1020.0, 1030.0, -1015.0, -1030.0))
def test_gradient_from_a_kept_lse_of_rows_far_from_zero(B, base, dtype, n, k):
    if not _fits(base, dtype):
        base = math.copysign(4e4, base)
    _check_kept(B, *_rows(base, dtype, n, k), 1.0)


@pytest.mark.parametrize("n,k", SIZES)
@pytest.mark.parametrize("dtype", LOGITS)
@pytest.mark.parametrize("tau,base,spread", TEMPERATURES)
def test_gradient_from_a_kept_lse_at_temperatures(B, tau, base, spread, dtype, n, k):
    _check_kept(B, *_rows(base, dtype, n, k, spread), tau)


@pytest.mark.parametrize("n", [500, 50_000])
def test_gradient_from_a_kept_lse_of_rows_that_are_nan(B, n):
    """Rows with NaN or infinity, and rows whose lse is one; their neighbours are not touched by it."""
    logits = torch.randn((6, n), generator=_gen(n), device="cuda") * 2000
    ids = torch.zeros((6, 1), dtype=torch.int32, device="cuda")
    z = torch.zeros((6, 1), device="cuda")
    logits[0, 3], logits[1, 3], logits[2] = math.nan, math.inf, -math.inf
    lse = B.spsyrk_distill(logits, ids, z)[1]
    lse[4] = math.nan
    grad = B.spsyrk_distill_grad(logits, lse, ids, z)
    assert grad[[0, 1, 2, 4]].isnan().all() and not grad[[3, 5]].isnan().any()


@pytest.mark.parametrize("norm", [800.0, 1e5, math.inf])
def test_a_norm_that_leaves_the_teacher_nothing(B, norm):
    """p = 0 for every entry: nothing is added, not for q = 0 either; NaN among the logits is NaN all the same."""
    logits = torch.zeros((6, 40), device="cuda")
    logits[1, 1] = -math.inf
    logits[2, 7], logits[3] = math.nan, -math.inf
    ids = torch.tensor([[1, 2]] * 6, dtype=torch.int32, device="cuda")
    z = torch.zeros((6, 2), device="cuda")
    z[4, 1] = math.nan
    z[5] = -math.inf
    loss, lse, grad = B.spsyrk_distill(logits, ids, z, teacher_lse=torch.full((6,), norm, device="cuda"), grad=True)
    assert (loss[[0, 1, 5]] == 0).all() and (grad[[0, 1, 5]] == 0).all()
    assert loss[2:5].isnan().all() and grad[2:5].isnan().all()


@pytest.mark.parametrize("m,n,k", [(950, 3157, 256), (16, 7000, 256), (300, 7000, 120), (64, 333, 30)])
@pytest.mark.parametrize("base", [3.0, -500.0, -2000.0, 2700.0, -7000.0])
@pytest.mark.parametrize("dtype", LOGITS)
def test_the_same_call_gives_the_same_bits(B, dtype, base, m, n, k):
    """Rows whose units and teacher's entries do not fill the last turn of a warp, ids that occur twice: every repetition, right and alike."""
    gen = _gen(n + k)
    for spread in (0.0, 1.0):
        logits = (base + spread * torch.randn((m, n), generator=gen, device="cuda")).to(dtype)
        ids = torch.randint(0, n // 2, (m, k), generator=gen, device="cuda", dtype=torch.int32)
        z = (base + torch.randn((m, k), generator=gen, device="cuda")).to(dtype)
        first = None
        for _ in range(40):
            loss, lse, grad = B.spsyrk_distill(logits, ids, z, grad=True)
            out = (loss, lse, grad, B.spsyrk_distill_grad(logits, lse, ids, z))
            first = first or [t.clone() for t in out]
            assert all(torch.equal(a, b) for a, b in zip(out, first))
        # (double precision over all rows at once; a row's q is at most one: 2^-9 of it and of p, and the steps of the type's smallest numbers)
        logp = torch.log_softmax(z.double(), 1)
        expected = torch.softmax(logits.double(), 1).scatter_add_(1, ids.long(), -logp.exp())
        size = torch.softmax(logits.double(), 1).scatter_add_(1, ids.long(), logp.exp())
        assert ((first[2].double() - expected).abs() <= size * (torch.finfo(dtype).eps / 2 + 2.0 ** -12) + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps).all()
