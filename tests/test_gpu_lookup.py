"""Lookups and their gradients against the definition in double precision: every type, odd widths and strides, rows of any length,
padding, ids that occur often."""
import pytest
import torch

import vocabulary as V

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_09713_b200 import binding
    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _ids(count, n, gen, skew=False, padding=0.1):
    if skew:
        ids = (n * torch.rand(count, generator=gen, device="cuda") ** 8).to(torch.int32)
    else:
        ids = torch.randint(0, max(n, 1), (count,), generator=gen, device="cuda", dtype=torch.int32)
    for k, pad in enumerate(V.PADDING + (n,)):
        ids[torch.rand(count, generator=gen, device="cuda") < padding / 5] = pad
    return ids


def _weights(count, dtype, gen):
    w = torch.randn(count, generator=gen, device="cuda", dtype=torch.float64)
    return w.to(torch.float64 if dtype == torch.float64 else torch.float32)


LENGTHS = {
    "short": [0, 1, 2, 0, 7, 8, 9, 16, 17, 0],
    "long": [0, 700, 3, 129, 0, 2100, 1],
    "one": [300],
    "none": [0, 0, 0],
    "many": [(i * 7) % 23 for i in range(700)],
    "many with long ones": [(i * 7) % 23 for i in range(300)] + [3000, 0, 515] + [5] * 30,
}


def _rowptr(lengths, before=0):
    return torch.tensor([before] + lengths, device="cuda").cumsum(0)


# (rows or lengths, ids of a row or None for row pointers, n, p, elements between rows, offset into the buffer)
SHAPES = [
    (1, 1, 1, 1, 0, 0), (16, 1, 300, 1024, 0, 0), (1000, 1, 77, 64, 8, 0), (333, 1, 200, 1001, 0, 0), (40, 1, 50, 4096, 0, 1), (20_000, 1, 100, 72, 0, 0),
    (9, 1, 10, 5, 3, 0), (3, 1, 2, 9000, 0, 0), (50, 3, 60, 64, 0, 0), (7, 200, 90, 33, 1, 0), (300, 40, 500, 256, 0, 0), (2, 1500, 400, 136, 0, 0),
    (333, 1, 200, 1002, 0, 0), (50, 5, 90, 70, 0, 2), (40, 1, 50, 30, 4, 0), ("short", None, 30, 66, 0, 0), ("long", None, 200, 502, 0, 0),
    ("short", None, 30, 64, 0, 0), ("long", None, 500, 7, 0, 0), ("long", None, 300, 520, 8, 8), ("one", None, 20, 2000, 0, 0), ("none", None, 9, 16, 0, 0),
    ("many", None, 1000, 48, 0, 0), ("many with long ones", None, 400, 100, 0, 0), ("many", None, 3, 1, 0, 0),
]


def _case(shape, dtype, weighted, seed=1):
    rows, k, n, p, pad, offset = shape
    gen = _gen(seed)
    rowptr = None if k else _rowptr(LENGTHS[rows])
    m, count = (rows, rows * k) if k else (len(LENGTHS[rows]), int(rowptr[-1]))
    ids = _ids(count, n, gen, skew=weighted)
    w = _weights(count, dtype, gen) if weighted else None
    if k and k > 1:
        ids, w = ids.view(m, k), None if w is None else w.view(m, k)
    return m, n, p, ids, w, rowptr, gen


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", V.DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_lookup(B, shape, dtype, weighted):
    pad, offset = shape[4:]
    m, n, p, ids, w, rowptr, gen = _case(shape, dtype, weighted)
    e, _ = V.matrix(n, p, dtype, gen, pad, offset)
    y, buffer = V.matrix(m, p, dtype, gen, pad, offset)
    between = buffer.clone()
    between[offset:].view(m, p + pad)[:, :p] = 0
    B.spsyrk_lookup(ids, e, rowptr=rowptr, weights=w, scale=1.7, y=y)
    V.check_lookup(y, ids, e, rowptr, w, 1.7)
    first = y.clone()
    buffer[offset:].view(m, p + pad)[:, :p] = 0
    assert torch.equal(buffer, between)  # what lies between the rows is as it was
    again = B.spsyrk_lookup(ids, e.contiguous(), rowptr=rowptr, weights=w, scale=1.7)  # (rows that may lie otherwise)
    V.check_lookup(again, ids, e, rowptr, w, 1.7)
    B.spsyrk_lookup(ids, e, rowptr=rowptr, weights=w, scale=1.7, y=y)
    assert torch.equal(y, first)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("dtype", V.DTYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_gradients(B, shape, dtype, weighted):
    pad, offset = shape[4:]
    m, n, p, ids, w, rowptr, gen = _case(shape, dtype, weighted, 2)
    dy, _ = V.matrix(m, p, dtype, gen, pad, offset)
    kinds = (dtype,) if dtype in (torch.float64, torch.float32) else (dtype, torch.float32)
    for g in kinds:
        de = B.spsyrk_lookup_grad(ids, dy, n, rowptr=rowptr, weights=w, scale=-0.6, dtype=g)
        assert de.dtype == g
        V.check_grad(de, ids, dy, rowptr, w, -0.6)
        assert torch.equal(de, B.spsyrk_lookup_grad(ids, dy, n, rowptr=rowptr, weights=w, scale=-0.6, dtype=g))
        # added to what is there, between other things
        old, buffer = V.matrix(n, p, g, gen, pad, offset)
        kept = buffer.clone()
        before = old.clone()
        B.spsyrk_lookup_grad(ids, dy, n, rowptr=rowptr, weights=w, scale=-0.6, de=old, accumulate=True)
        V.check_grad(old, ids, dy, rowptr, w, -0.6, before)
        absent = torch.ones(n, dtype=torch.bool, device="cuda")
        flat, row = ids.reshape(-1).long(), V.rows_of(rowptr, m, ids.numel())
        absent[flat[(flat >= 0) & (flat < n) & (row >= 0)]] = False
        assert torch.equal(old[absent], before[absent])
        old.copy_(before)
        assert torch.equal(buffer, kept)
        B.spsyrk_lookup_grad(ids, dy, n, rowptr=rowptr, weights=w, scale=-0.6, de=old)
        assert torch.equal(old, de)
        old.copy_(before)
        assert torch.equal(buffer, kept)
    e, _ = V.matrix(n, p, dtype, gen, pad, offset)
    V.check_grad_weights(B.spsyrk_lookup_grad_weights(ids, e, dy, rowptr=rowptr, scale=2.5), ids, e, dy, rowptr, 2.5)


@pytest.mark.parametrize("weighted", [False, True])
@pytest.mark.parametrize("count,n,p", [(6144, 300, 40), (6145, 300, 40), (8193, 255, 16), (8193, 256, 16), (6100, 100_000, 33), (30_000, 70_000, 24), (100_001, 1, 65),
                                       (50_000, 3, 128), (40_000, 600, 7), (5000, 1, 512), (70_000, 20, 1000)])
def test_gradient_of_ids_that_occur_often(B, count, n, p, weighted):
    gen = _gen(count + n)
    ids = _ids(count, n, gen, skew=True)
    w = _weights(count, torch.float32, gen) if weighted else None
    dy, _ = V.matrix(count, p, torch.bfloat16, gen)
    de = B.spsyrk_lookup_grad(ids, dy, n, weights=w, scale=0.5, dtype=torch.float32)
    flat = ids.long()
    held = (flat >= 0) & (flat < n)
    x = dy.double() * (1.0 if w is None else w.double()[:, None]) * 0.5
    expected, size = (torch.zeros((n, p), dtype=torch.float64, device="cuda").index_add_(0, flat[held], t[held]) for t in (x, x.abs()))
    often = torch.bincount(flat[held], minlength=n)[:, None]
    V.check(de, expected, (often + 6) * 2.0 ** -24 * size + V.half_step(de.dtype, expected))
    assert torch.equal(de, B.spsyrk_lookup_grad(ids, dy, n, weights=w, scale=0.5, dtype=torch.float32))


def test_values_of_padded_places_are_not_looked_at(B):
    gen = _gen(5)
    nan, inf = float("nan"), float("inf")
    e, _ = V.matrix(40, 24, torch.float32, gen)
    e[7], e[8] = nan, inf
    ids = torch.tensor([[1, -1, 2], [-1, -1, -1], [40, 3, 3], [5, 6, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")
    w = torch.ones((4, 3), device="cuda")
    w[0, 1] = w[1, 0] = w[2, 0] = nan
    w[3, 2] = inf
    y = B.spsyrk_lookup(ids, e, weights=w)
    V.check_lookup(y, ids, e.nan_to_num(0.0, 0.0, 0.0), None, torch.ones_like(w), 1.0)  # (the plain form multiplies by all rows)
    assert torch.equal(y[1], torch.zeros_like(y[1]))
    dy, _ = V.matrix(4, 24, torch.float32, gen)
    dy[1] = nan  # only padded places
    de = B.spsyrk_lookup_grad(ids, dy, 40, weights=w)
    ones = torch.ones_like(w)
    V.check_grad(de, ids, torch.where(torch.isnan(dy), 0.0, dy), None, ones, 1.0)
    dw = B.spsyrk_lookup_grad_weights(ids, e, dy)
    assert torch.equal(dw == 0, (ids < 0) | (ids >= 40))
    # NaN in the table reaches the rows that name it, and no others
    y = B.spsyrk_lookup(torch.tensor([7, 8, 9], dtype=torch.int32, device="cuda"), e)
    assert torch.isnan(y[0]).all() and torch.isinf(y[1]).all() and torch.equal(y[2], e[9])


def test_entries_of_no_row(B):
    """Buffers longer than their rows: what stands before the first row and behind the last one is nobody's."""
    for lengths, before, behind in (([3, 0, 5], 4, 6), ([2] * 3000, 100, 5000), ([900, 2], 1, 2)):
        gen = _gen(behind)
        rowptr = _rowptr(lengths, before)
        count = before + sum(lengths) + behind
        ids, w = _ids(count, 50, gen), _weights(count, torch.float32, gen)
        e, _ = V.matrix(50, 36, torch.float32, gen)
        dy, _ = V.matrix(len(lengths), 36, torch.float32, gen)
        V.check_lookup(B.spsyrk_lookup(ids, e, rowptr=rowptr, weights=w), ids, e, rowptr, w, 1.0)
        V.check_grad(B.spsyrk_lookup_grad(ids, dy, 50, rowptr=rowptr, weights=w), ids, dy, rowptr, w, 1.0)
        V.check_grad_weights(B.spsyrk_lookup_grad_weights(ids, e, dy, rowptr=rowptr), ids, e, dy, rowptr, 1.0)


def test_no_rows_but_entries(B):
    rowptr, ids = torch.tensor([3], device="cuda"), torch.arange(5, dtype=torch.int32, device="cuda")
    e, dy = torch.ones((9, 8), device="cuda"), torch.ones((0, 8), device="cuda")
    assert B.spsyrk_lookup(ids, e, rowptr=rowptr).shape == (0, 8)
    de = torch.ones((9, 8), device="cuda")
    B.spsyrk_lookup_grad(ids, dy, 9, rowptr=rowptr, de=de, accumulate=True)
    assert (de == 1).all()
    assert (B.spsyrk_lookup_grad(ids, dy, 9, rowptr=rowptr) == 0).all()
    assert (B.spsyrk_lookup_grad_weights(ids, e, dy, rowptr=rowptr) == 0).all()


@pytest.mark.parametrize("m,k,p", [(300, 900, 64), (300, 900, 20), (257, 130, 8), (1000, 600, 16), (3, 20_000, 100), (400, 33, 2000)])
def test_rows_of_every_way(B, m, k, p):
    """Shared by the groups of a warp, by clusters, one group each: fixed and ragged rows."""
    gen = _gen(m + k)
    ids, w = _ids(m * k, 5000, gen), _weights(m * k, torch.float32, gen)
    e, _ = V.matrix(5000, p, torch.float32, gen)
    V.check_lookup(B.spsyrk_lookup(ids.view(m, k), e, weights=w.view(m, k)), ids, e, torch.arange(m + 1, device="cuda") * k, w, 1.0)
    length = torch.randint(0, 2 * k, (m,), generator=gen, device="cuda").cumsum(0)
    rowptr = torch.cat((torch.zeros(1, dtype=torch.int64, device="cuda"), length)).clamp(max=m * k)
    V.check_lookup(B.spsyrk_lookup(ids, e, rowptr=rowptr, weights=w), ids, e, rowptr, w, 1.0)


def test_nothing_to_do(B):
    none = torch.empty(0, dtype=torch.int32, device="cuda")
    for dtype in V.DTYPES:
        e = torch.ones((5, 8), dtype=dtype, device="cuda")
        assert B.spsyrk_lookup(none, e).shape == (0, 8)
        assert torch.equal(B.spsyrk_lookup(none.view(3, 0), e), torch.zeros((3, 8), dtype=dtype, device="cuda"))
        assert B.spsyrk_lookup(torch.tensor([1, -1], dtype=torch.int32, device="cuda"), e[:, :0]).shape == (2, 0)
        assert torch.equal(B.spsyrk_lookup(torch.tensor([1, -1], dtype=torch.int32, device="cuda"), e[:0]), torch.zeros((2, 8), dtype=dtype, device="cuda"))
        de = torch.full((5, 10), 3.0, dtype=dtype, device="cuda")
        B.spsyrk_lookup_grad(none, e[:0], 5, de=de[:, :8], accumulate=True)
        assert (de == 3).all()
        B.spsyrk_lookup_grad(none, e[:0], 5, de=de[:, :8])
        assert (de[:, :8] == 0).all() and (de[:, 8:] == 3).all()
        assert B.spsyrk_lookup_grad(torch.tensor([0], dtype=torch.int32, device="cuda"), e[:1], 0).shape == (0, 8)
        all_padding = torch.full((4,), -1, dtype=torch.int32, device="cuda")
        assert (B.spsyrk_lookup_grad(all_padding, e[:4], 5) == 0).all()
        assert B.spsyrk_lookup_grad_weights(none, e, e[:0]).shape == (0,)


def test_gradients_are_those_of_differences(B):
    """(f(x + h d) - f(x - h d)) / 2h = <gradient, d>, exactly for a function that is linear in x, f = <lookup, dY>."""
    gen = _gen(9)
    rowptr = _rowptr(LENGTHS["short"])
    count, n, p = int(rowptr[-1]), 12, 10
    ids, w = _ids(count, n, gen), _weights(count, torch.float64, gen)
    e, _ = V.matrix(n, p, torch.float64, gen)
    dy, _ = V.matrix(len(LENGTHS["short"]), p, torch.float64, gen)
    f = lambda e, w: (B.spsyrk_lookup(ids, e, rowptr=rowptr, weights=w, scale=3.0) * dy).sum()
    de = B.spsyrk_lookup_grad(ids, dy, n, rowptr=rowptr, weights=w, scale=3.0)
    dw = B.spsyrk_lookup_grad_weights(ids, e, dy, rowptr=rowptr, scale=3.0)
    for _ in range(5):
        d, t = torch.randn(e.shape, generator=gen, device="cuda", dtype=torch.float64), torch.randn(w.shape, generator=gen, device="cuda", dtype=torch.float64)
        for change, slope in ((f(e + d, w) - f(e - d, w), (de * d).sum()), (f(e, w + t) - f(e, w - t), (dw * t).sum())):
            # about 2000 products of values around one: 2000 * 2^-53 * a few thousand
            assert abs(float(change / 2 - slope)) < 1e-9


def test_offsets_beyond_32_bits(B):
    """A table of more than 2^31 elements, and its gradient."""
    n, p = 1_100_000, 2048
    gen = _gen(11)
    ids = torch.tensor([n - 1, 0, n - 2, -1, n - 1, 1_050_001], dtype=torch.int32, device="cuda")
    e = torch.zeros((n, p), dtype=torch.bfloat16, device="cuda")
    e[ids[ids >= 0].long()] = torch.randn((5, p), generator=gen, device="cuda").bfloat16()
    y = B.spsyrk_lookup(ids, e)
    assert torch.equal(y[ids >= 0], e[ids[ids >= 0].long()]) and (y[3] == 0).all()
    dy, _ = V.matrix(6, p, torch.bfloat16, gen)
    assert torch.equal(B.spsyrk_lookup_grad_weights(ids, e, dy)[[1]], B.spsyrk_lookup_grad_weights(ids[[1]], e, dy[[1]]))
    de = e.fill_(5.0)
    B.spsyrk_lookup_grad(ids, dy, n, de=de)
    assert torch.equal(de[n - 2], dy[2]) and torch.equal(de[0], dy[1]) and torch.equal(de[1_050_001], dy[5])
    assert torch.equal(de[n - 1], (dy[0].float() + dy[4].float()).bfloat16())
    assert int((de != 0).any(1).sum()) == 4


@pytest.mark.parametrize("pad", [0, 4])
@pytest.mark.parametrize("count", [100, 7000])
def test_few_entries_of_a_large_matrix(B, count, pad):
    """More than 256 MB with few rows of entries: cleared as a whole; what lies between the rows stays."""
    n, p = 70_000, 1000
    gen = _gen(count)
    ids = _ids(count, n, gen)
    dy, _ = V.matrix(count, p, torch.float32, gen)
    de = torch.full((n, p + pad), 7.0, device="cuda")
    B.spsyrk_lookup_grad(ids, dy, n, de=de[:, :p])
    held = (ids >= 0) & (ids < n)
    expected, size = (torch.zeros((n, p), dtype=torch.float64, device="cuda").index_add_(0, ids[held].long(), t[held]) for t in (dy.double(), dy.double().abs()))
    often = torch.bincount(ids[held].long(), minlength=n)[:, None]
    V.check(de[:, :p], expected, (often + 6) * 2.0 ** -24 * size + V.half_step(de.dtype, expected))
    assert (de[:, p:] == 7).all()


@pytest.mark.parametrize("count", [700, 9000])
def test_streams_and_graphs(B, count):
    gen = _gen(count)
    n, p, k = 500, 200, 4
    ids, w = _ids(count * k, n, gen, skew=True).view(count, k), _weights(count * k, torch.float32, gen).view(count, k)
    e, _ = V.matrix(n, p, torch.float32, gen)
    dy, _ = V.matrix(count, p, torch.float32, gen)
    call = lambda stream=None: (B.spsyrk_lookup(ids, e, weights=w, stream=stream), B.spsyrk_lookup_grad(ids, dy, n, weights=w, stream=stream),
                                B.spsyrk_lookup_grad_weights(ids, e, dy, stream=stream))
    expected = call()
    streams = [torch.cuda.Stream() for _ in range(3)]
    torch.cuda.synchronize()
    results = [call(s) for s in streams for _ in range(2)]  # side by side, each with a workspace of its own
    torch.cuda.synchronize()
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(r, expected))
    with torch.cuda.stream(streams[0]):
        call()
    torch.cuda.current_stream().wait_stream(streams[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for shift in (0, 1):  # replayed for other ids in the same place
        ids.copy_(torch.where(ids >= 0, (ids + shift) % n, ids))
        for t in out:
            t.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, call()))
