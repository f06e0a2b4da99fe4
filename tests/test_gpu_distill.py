"""Distillation from a teacher's top logits against the definition in double precision: every type, odd vocabularies and strides, rows
without entries, masked logits, ids that a row holds twice, rows of more entries than shared memory takes."""
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


def _teacher(count, n, gen, dtype, padding=0.05):
    ids = torch.randint(0, n, (count,), generator=gen, device="cuda", dtype=torch.int32)
    for pad in V.PADDING + (n,):
        ids[torch.rand(count, generator=gen, device="cuda") < padding / 5] = pad
    return ids, (3 * torch.randn(count, generator=gen, device="cuda")).to(dtype)


def _copy(logits):
    """A copy that lies to 16-byte boundaries as the original does: sums are the same bits for the same alignment."""
    offset = logits.data_ptr() % 16 // logits.element_size()
    m, ld = logits.shape[0], max(logits.stride(0), logits.shape[1])
    out = torch.zeros(offset + m * ld, dtype=logits.dtype, device="cuda")[offset:].view(m, ld)[:, :logits.shape[1]]
    return out.copy_(logits)


def _run(B, logits, ids, teacher, **kw):
    """In one call and in two, beside the logits and in their place: (loss, lse, gradient, gradient from the lse of the call without)."""
    loss, lse, grad = B.spsyrk_distill(logits, ids, teacher, grad=True, **kw)
    loss2, lse = B.spsyrk_distill(logits, ids, teacher, **kw)
    assert torch.equal(loss.isnan(), loss2.isnan())
    kept = B.spsyrk_distill_grad(logits, lse, ids, teacher, **kw)
    inside = _copy(logits)
    both = B.spsyrk_distill(inside, ids, teacher, grad=inside, **kw)
    assert both[2] is inside and torch.equal(inside.nan_to_num(), grad.nan_to_num()) and torch.equal(both[0].nan_to_num(), loss.nan_to_num())
    inside = _copy(logits)
    B.spsyrk_distill_grad(inside, lse, ids, teacher, grad=inside, **kw)
    assert torch.equal(inside.nan_to_num(), kept.nan_to_num())
    return loss, lse, grad, kept


def _check(B, logits, ids, teacher, rowptr=None, teacher_lse=None, row_weights=None, tau=1.0):
    kw = dict(rowptr=rowptr, teacher_lse=teacher_lse, row_weights=row_weights, temperature=tau)
    loss, lse, grad, kept = _run(B, logits, ids, teacher, **kw)
    V.check_distill((loss, lse, kept), logits, ids, teacher, rowptr, teacher_lse, row_weights, tau)
    loss, lse, grad = B.spsyrk_distill(logits, ids, teacher, grad=grad, **kw)
    V.check_distill((loss, lse, grad), logits, ids, teacher, rowptr, teacher_lse, row_weights, tau)
    loss = B.spsyrk_distill(logits, ids, teacher, **kw)[0]
    V.check_distill((loss, None, None), logits, ids, teacher, rowptr, teacher_lse, row_weights, tau)
    return loss, lse, grad


# rows, entries of a row, n, elements between rows, offset, temperature
FIXED = [(1, 1, 1, 0, 0, 1.0), (3, 2, 7, 0, 0, 2.0), (17, 16, 1000, 24, 0, 1.0), (5, 40, 1001, 0, 1, 0.5), (300, 8, 515, 2, 3, 1.5), (2, 500, 40_001, 0, 0, 3.0),
         (150, 30, 16_384, 0, 0, 1.0), (1, 64, 131_072, 0, 0, 1.0), (20, 1024, 2900, 0, 0, 1.0), (4, 1025, 9000, 7, 0, 2.0), (2, 5000, 100_003, 0, 0, 1.0), (9, 0, 50, 0, 0, 1.0),
         (2, 9, 1_500_001, 0, 0, 1.0), (1, 3000, 700_000, 0, 0, 1.0), (1000, 5, 300, 0, 0, 1.0), (900, 6, 4096, 8, 0, 1.0), (450, 3, 20_000, 0, 0, 1.0)]


@pytest.mark.parametrize("dtype", LOGITS)
@pytest.mark.parametrize("shape", FIXED, ids=str)
def test_fixed_number_of_entries(B, shape, dtype):
    m, k, n, pad, offset, tau = shape
    gen = _gen(n + m)
    logits, buffer = V.matrix(m, n, dtype, gen, pad, offset, spread=3.0)
    ids, z = _teacher(m * k, n, gen, dtype)
    before = buffer.clone()
    _check(B, logits, ids.view(m, k), z.view(m, k), tau=tau)
    assert torch.equal(buffer, before)


@pytest.mark.parametrize("teacher_dtype", LOGITS)
@pytest.mark.parametrize("dtype", LOGITS)
def test_ragged_rows_weights_and_a_given_norm(B, dtype, teacher_dtype):
    lengths = [0, 1, 5, 1023, 0, 1024, 1100, 64, 2, 3, 0, 30, 31]
    rowptr = torch.tensor([2] + lengths, device="cuda").cumsum(0)
    m, n, count = len(lengths), 2003, 2 + sum(lengths) + 9
    gen = _gen(3)
    logits, _ = V.matrix(m, n, dtype, gen, 1, 0, spread=2.0)
    ids, z = _teacher(count, n, gen, teacher_dtype)
    r = torch.randn(m, generator=gen, device="cuda")
    r[2] = r[7] = 0.0
    lse = torch.full((m,), 12.0, device="cuda") + torch.rand(m, generator=gen, device="cuda")
    for kw in (dict(), dict(row_weights=r), dict(teacher_lse=lse), dict(row_weights=r, teacher_lse=lse, tau=1.7), dict(teacher_lse=lse + 28.0, tau=0.5)):
        loss, norm, grad = _check(B, logits, ids, z, rowptr=rowptr, **kw)
        out = torch.tensor(lengths, device="cuda") == 0
        if "row_weights" in kw:
            out |= r == 0
        assert (loss[out] == 0).all() and (norm[out] == 0).all() and (grad[out] == 0).all()


@pytest.mark.parametrize("entries", [6, 200, 1024, 1500, 4000])
def test_an_id_that_a_row_holds_more_than_once(B, entries):
    gen = _gen(entries)
    n, m = 2999, 4
    logits, _ = V.matrix(m, n, torch.float32, gen)
    ids, z = _teacher(m * entries, n, gen, torch.float32)
    ids = (ids % 37).view(m, entries)  # few ids, each many times
    ids[3] = 2998
    _check(B, logits, ids, z.view(m, entries))
    first = B.spsyrk_distill(logits, ids, z.view(m, entries), grad=True)
    for _ in range(3):
        assert all(torch.equal(a, b) for a, b in zip(first, B.spsyrk_distill(logits, ids, z.view(m, entries), grad=True)))


@pytest.mark.parametrize("n", [64, 70_000])
@pytest.mark.parametrize("dtype", LOGITS)
def test_masked_logits(B, dtype, n):
    """-infinity and the type's lowest value at ids that are not the teacher's, one logit far above the rest, a row of lowest values."""
    gen = _gen(n)
    lowest = torch.finfo(dtype).min
    logits, _ = V.matrix(6, n, dtype, gen)
    ids = torch.tensor([[1, 2, 3]] * 6, dtype=torch.int32, device="cuda")
    z = torch.randn((6, 3), generator=gen, device="cuda").to(dtype)
    logits[0, 5:] = -math.inf
    logits[1, 5:] = lowest
    logits[2, 10] = 60.0 if dtype == torch.float16 else 80.0
    z[3] = lowest
    z[4, 1] = -math.inf
    z[5, 0] = lowest
    _check(B, logits, ids, z)
    # nothing but the lowest value: q is the same everywhere
    logits[2] = lowest
    V.check_distill(B.spsyrk_distill(logits, ids, z, grad=True), logits, ids, z)


@pytest.mark.parametrize("n", [500, 50_000])
def test_infinities_and_nan(B, n):
    nan, inf = math.nan, math.inf
    gen = _gen(n)
    m = 9
    logits, _ = V.matrix(m, n, torch.float32, gen)
    ids = torch.tensor([[1, n - 1]] * m, dtype=torch.int32, device="cuda")
    z = torch.randn((m, 2), generator=gen, device="cuda")
    w = torch.ones(m, device="cuda")
    logits[0, 7], logits[1, 7], logits[2] = nan, inf, -inf   # the whole row is NaN
    z[3, 0], z[4, 1] = nan, inf                              # of the teacher's too
    logits[5] = nan                                          # left out by its weight, by having no teacher
    w[5] = 0.0
    logits[6] = inf
    z[6] = -inf
    logits[7, 1] = -inf                                      # q = 0 where p > 0: the loss is infinite, the gradient -p
    loss, lse, grad, kept = _run(B, logits, ids, z, row_weights=w)
    assert torch.equal(loss.isnan(), torch.arange(m, device="cuda") < 5)
    for g in (grad, kept):
        assert g[:5].isnan().all() and not g[5:].isnan().any()
        assert (g[5:7] == 0).all() and (loss[5:7] == 0).all()
    assert loss[7] == inf
    p = torch.softmax(z[7].double(), 0)
    assert abs(float(grad[7, 1]) + float(p[0])) < 2.0 ** -20
    V.check_distill((loss[8:], lse[8:], grad[8:]), logits[8:], ids[8:], z[8:])


def test_lse_and_gradient_of_infinite_rows_stay_in_their_rows(B):
    logits = torch.zeros((3, 40), device="cuda")
    logits[1] = math.nan
    ids = torch.zeros((3, 1), dtype=torch.int32, device="cuda")
    loss, lse, grad = B.spsyrk_distill(logits, ids, torch.zeros((3, 1), device="cuda"), grad=True)
    for i in (0, 2):
        V.check_distill((loss[[i]], lse[[i]], grad[[i]]), logits[[i]], ids[[i]], torch.zeros((1, 1), device="cuda"))


def test_gradient_is_that_of_differences(B):
    """Central differences of the loss in double precision agree with the gradient, and so does the kernel's loss with that loss."""
    gen = _gen(21)
    n, m, k, tau = 60, 3, 5, 2.0
    logits, _ = V.matrix(m, n, torch.float32, gen)
    ids, z = _teacher(m * k, n, gen, torch.float32, padding=0.0)
    ids, z = ids.view(m, k), z.view(m, k)
    loss, _, grad = B.spsyrk_distill(logits, ids, z, temperature=tau, grad=True)
    for _ in range(4):
        d = torch.randn((m, n), generator=gen, device="cuda", dtype=torch.float64)
        f = lambda s: V.distill_plain(s, ids, z, None, None, None, tau, tau * tau)[0][0].sum()
        h = 1e-4
        slope = float(f(logits.double() + h * d) - f(logits.double() - h * d)) / (2 * h)
        # third derivatives of log sum exp along d are below 10 |d|^3, their share h^2 / 6 of that; the gradient's own error: 1e-5 of it
        assert abs(slope - float((grad.double() * d).sum())) < 1e-5 * float((grad.double() * d).abs().sum()) + 2e-8 * float(d.abs().max()) ** 3 * m * 10


def test_offsets_beyond_32_bits(B):
    m, n = 17_000, 131_072
    logits = torch.zeros((m, n), dtype=torch.bfloat16, device="cuda")
    last = slice(m - 3, m)
    logits[last] = torch.randn((3, n), generator=_gen(1), device="cuda").bfloat16()
    ids = torch.full((m, 2), n - 1, dtype=torch.int32, device="cuda")
    ids[:, 0] = 3
    z = torch.zeros((m, 2), device="cuda")
    w = torch.zeros(m, device="cuda")
    w[last] = 1.0
    loss, lse, grad = B.spsyrk_distill(logits, ids, z, row_weights=w, grad=True)
    V.check_distill((loss[last], lse[last], grad[last]), logits[last], ids[last], z[last])
    assert (loss[:-3] == 0).all() and not grad[:-3].any()


@pytest.mark.parametrize("m", [2, 400])
def test_streams_and_graphs(B, m):
    gen = _gen(m)
    n, k = 20_011, 30
    logits, _ = V.matrix(m, n, torch.bfloat16, gen)
    ids, z = _teacher(m * k, n, gen, torch.bfloat16)
    ids, z = ids.view(m, k), z.view(m, k)
    call = lambda stream=None: B.spsyrk_distill(logits, ids, z, grad=True, stream=stream)
    expected = call()
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for r in [call(s) for s in streams]:
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(r, expected))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
        kept = B.spsyrk_distill_grad(logits, out[1], ids, z)
    logits.copy_(-logits)
    graph.replay()
    torch.cuda.synchronize()
    expected = call()
    assert all(torch.equal(a, b) for a, b in zip(out, expected))
    assert torch.equal(kept, B.spsyrk_distill_grad(logits, expected[1], ids, z))
