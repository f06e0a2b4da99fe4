"""What the lookups and the distillation refuse, on the host: by the C entry points before they touch the device, by the binding
before it calls them; and launches that do not start are reported."""
import ctypes
import os
import subprocess
import sys

import pytest
import torch

import test_launch_errors as launches

F64, F32, I32, BF16, F16 = range(5)
INVALID, WORKSPACE, OVERFLOW = 1, 3, 4
AT = ctypes.c_void_p(4096)  # stands for a device pointer; a call that is refused does not look at it
MOST = 2 ** 31 - 1


@pytest.fixture(scope="module")
def lib():
    from paper_2608_09713_b200 import build
    return ctypes.CDLL(build.build_cuda())


def _call(function, defaults, kinds):
    def call(lib, **changes):
        assert not set(changes) - set(defaults)
        values = [changes.get(name, value) for name, value in defaults.items()]
        return getattr(lib, function)(*[kinds.get(type(v), lambda x: x)(v) for v in values], None)
    return call


KINDS = {int: ctypes.c_int64, float: ctypes.c_double}


class Code:  # an enumeration or a truth value: a C int
    def __init__(self, value):
        self.value = value


KINDS[Code] = lambda c: ctypes.c_int(c.value)

lookup = _call("spsyrk_lookup", dict(m=6, n=10, p=8, nnz=6, dtype=Code(F32), rowptr=None, ids=AT, weights=None, scale=1.0, e=AT, lde=8, y=AT, ldy=8), KINDS)
grad_weights = _call("spsyrk_lookup_grad_weights", dict(m=6, n=10, p=8, nnz=6, dtype=Code(F32), rowptr=None, ids=AT, scale=1.0, e=AT, lde=8, dy=AT, lddy=8, dw=AT), KINDS)
distill = _call("spsyrk_distill", dict(m=6, n=10, nnz=12, dtype=Code(F32), tdtype=Code(F32), rowptr=None, ids=AT, teacher=AT, tlse=None, weights=None, tau=1.0,
                                       scale=1.0, logits=AT, ldl=10, loss=AT, lse=AT, grad=None, ldg=0), KINDS)
distill_grad = _call("spsyrk_distill_grad", dict(m=6, n=10, nnz=12, dtype=Code(F32), tdtype=Code(F32), rowptr=None, ids=AT, teacher=AT, tlse=None, weights=None,
                                                 tau=1.0, scale=1.0, logits=AT, ldl=10, lse=AT, grad=AT, ldg=10), KINDS)


def lookup_grad(lib, ws=None, nbytes=None, **changes):
    size = ctypes.c_size_t(0 if nbytes is None else nbytes)
    call = _call("spsyrk_lookup_grad", dict(m=6, n=10, p=8, nnz=6, dtype=Code(F32), gdtype=Code(F32), rowptr=None, ids=AT, weights=None, scale=1.0, dy=AT, lddy=8,
                                            de=AT, ldde=8, accumulate=Code(0), ws=ws, size=ctypes.byref(size)), KINDS)
    return call(lib, **changes), size.value


@pytest.mark.parametrize("call", [lookup, grad_weights])
def test_lookups_refuse(lib, call):
    other = "ldy" if call is lookup else "lddy"
    for changes in (dict(m=-1, nnz=0), dict(n=-1), dict(p=-1), dict(nnz=-1), dict(dtype=Code(I32)), dict(dtype=Code(5)), dict(dtype=Code(-1)), dict(lde=7),
                    {other: 7}, dict(ids=None), dict(e=None), {"y" if call is lookup else "dw": None}, dict(nnz=7), dict(m=0)):
        assert call(lib, **changes) == INVALID, changes
    for changes in (dict(m=MOST, nnz=0), dict(n=MOST), dict(nnz=MOST), dict(p=(1 << 21) + 1, lde=1 << 23, **{other: 1 << 23})):
        assert call(lib, **changes) == OVERFLOW, changes
    if call is lookup:
        assert call(lib, m=0, nnz=0) == 0 and call(lib, p=0) == 0
    else:
        assert call(lib, nnz=0) == 0


def test_lookup_grad_refuses(lib):
    status, size = lookup_grad(lib)
    assert status == 0 and size > 0
    assert lookup_grad(lib, nnz=100_000, m=100_000)[1] > 100_000 * 24
    for changes in (dict(m=-1), dict(n=-1), dict(p=-1), dict(nnz=-1), dict(dtype=Code(I32)), dict(gdtype=Code(BF16)), dict(gdtype=Code(F64)),
                    dict(dtype=Code(F64)), dict(dtype=Code(BF16), gdtype=Code(F16))):
        assert lookup_grad(lib, **changes)[0] == INVALID, changes
    for changes in (dict(m=MOST), dict(n=MOST), dict(nnz=MOST), dict(p=(1 << 21) + 1)):
        assert lookup_grad(lib, **changes)[0] == OVERFLOW, changes
    assert lookup_grad(lib, AT, size - 1)[0] == WORKSPACE
    assert lookup_grad(lib, ctypes.c_void_p(4097), size)[0] == INVALID
    for changes in (dict(lddy=7), dict(ldde=7), dict(ids=None), dict(dy=None), dict(de=None), dict(nnz=5), dict(m=0)):
        assert lookup_grad(lib, AT, 1 << 20, **changes)[0] == INVALID, changes
    assert lookup_grad(lib, AT, 1 << 20, n=0)[0] == 0 and lookup_grad(lib, AT, 1 << 20, p=0)[0] == 0
    i64 = ctypes.c_int64
    assert lib.spsyrk_lookup_grad(i64(6), i64(10), i64(8), i64(6), F32, F32, None, AT, None, ctypes.c_double(1), AT, i64(8), AT, i64(8), 0, AT, None, None) == INVALID


@pytest.mark.parametrize("call", [distill, distill_grad])
def test_distillation_refuses(lib, call):
    nan, inf = float("nan"), float("inf")
    for changes in (dict(m=-1, nnz=0), dict(n=-1), dict(nnz=-1), dict(dtype=Code(F64)), dict(dtype=Code(I32)), dict(dtype=Code(9)), dict(tdtype=Code(F64)),
                    dict(ldl=9), dict(grad=AT, ldg=9), dict(logits=AT, grad=AT, ldl=11, ldg=10), dict(ids=None), dict(teacher=None), dict(logits=None), dict(nnz=13),
                    dict(m=0), dict(tau=0.0), dict(tau=-1.0), dict(tau=nan), dict(tau=inf), dict(tau=1e-7), dict(tau=1e7)):
        assert call(lib, **changes) == INVALID, changes
    for changes in (dict(m=MOST, nnz=0), dict(n=MOST, ldl=MOST, ldg=MOST), dict(nnz=MOST)):
        assert call(lib, **changes) == OVERFLOW, changes
    assert call(lib, m=0, nnz=0) == 0
    if call is distill_grad:
        assert call(lib, lse=None) == INVALID and call(lib, grad=None) == INVALID


def test_the_binding_refuses():
    """Tensors on the host, of other types, shapes, strides: a ValueError, before anything is called."""
    from paper_2608_09713_b200 import binding as B
    ids, e = torch.zeros(4, dtype=torch.int32), torch.zeros((9, 8))
    z, logits, lse = torch.zeros((4, 2)), torch.zeros((4, 30)), torch.zeros(4)
    pairs = torch.zeros((4, 2), dtype=torch.int32)
    rowptr = torch.tensor([0, 2, 4])
    refused = [
        lambda: B.spsyrk_lookup(ids, e), lambda: B.spsyrk_lookup(ids.long(), e), lambda: B.spsyrk_lookup(ids, e.int()), lambda: B.spsyrk_lookup(ids, e[0]),
        lambda: B.spsyrk_lookup(ids, e.t()), lambda: B.spsyrk_lookup(ids, e[:1].expand(9, 8)), lambda: B.spsyrk_lookup(ids[::2], e),
        lambda: B.spsyrk_lookup(ids, e, weights=torch.zeros(3)), lambda: B.spsyrk_lookup(ids, e, weights=torch.zeros(4, dtype=torch.float64)),
        lambda: B.spsyrk_lookup(ids, e, rowptr=rowptr.int()), lambda: B.spsyrk_lookup(pairs, e, rowptr=rowptr), lambda: B.spsyrk_lookup(ids, e, rowptr=rowptr[:0]),
        lambda: B.spsyrk_lookup(ids, e, y=torch.zeros((3, 8))), lambda: B.spsyrk_lookup(ids, e, y=torch.zeros((4, 8), dtype=torch.bfloat16)),
        lambda: B.spsyrk_lookup(torch.zeros((2, 2, 1), dtype=torch.int32), e),
        lambda: B.spsyrk_lookup_grad(ids, e[:4], 9, accumulate=True), lambda: B.spsyrk_lookup_grad(ids, e, 9), lambda: B.spsyrk_lookup_grad(ids, e[:4], 9, dtype=torch.int32),
        lambda: B.spsyrk_lookup_grad(ids, e[:4], 9, de=torch.zeros((8, 8))), lambda: B.spsyrk_lookup_grad(ids, e[:4], 9),
        lambda: B.spsyrk_lookup_grad_weights(ids, e, e[:3]), lambda: B.spsyrk_lookup_grad_weights(ids, e, e[:4].bfloat16()),
        lambda: B.spsyrk_lookup_grad_weights(ids, e, e[:4], dw=torch.zeros(3)), lambda: B.spsyrk_lookup_grad_weights(ids, e, e[:4]),
        lambda: B.spsyrk_distill(logits, pairs, z), lambda: B.spsyrk_distill(logits.double(), pairs, z), lambda: B.spsyrk_distill(logits, pairs, z.double()),
        lambda: B.spsyrk_distill(logits, pairs, z[:3]), lambda: B.spsyrk_distill(logits[:3], pairs, z), lambda: B.spsyrk_distill(logits, pairs, z, row_weights=lse[:3]),
        lambda: B.spsyrk_distill(logits, pairs, z, teacher_lse=lse.double()), lambda: B.spsyrk_distill(logits, pairs, z, grad=torch.zeros((4, 29))),
        lambda: B.spsyrk_distill(logits, pairs, z, grad=torch.zeros((4, 30), dtype=torch.float16)),
        lambda: B.spsyrk_distill_grad(logits, lse[:3], pairs, z), lambda: B.spsyrk_distill_grad(logits, lse, pairs, z),
    ]
    for k, call in enumerate(refused):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(f"call {k} was not refused")


CALLS = r"""
import ctypes, sys
fake, lib = ctypes.CDLL(sys.argv[1]), ctypes.CDLL(sys.argv[2])
i64, f64, vp = ctypes.c_int64, ctypes.c_double, ctypes.c_void_p
fake.fake_launches.restype = ctypes.c_long
keep = []
def mem(n):
    keep.append(ctypes.create_string_buffer(n + 256))
    at = ctypes.addressof(keep[-1])
    return vp((at + 255) // 256 * 256)
big = mem(1 << 24)
def grad(m, nnz, rowptr, dtype, g):
    size = ctypes.c_size_t(0)
    call = lambda ws: lib.spsyrk_lookup_grad(i64(m), i64(70_000), i64(8), i64(nnz), dtype, g, rowptr, big, big, f64(1), big, i64(8), big, i64(8), 0, ws, ctypes.byref(size), None)
    assert call(None) == 0
    ws = mem(size.value)
    return lambda: call(ws)
lookup = lambda m, nnz, rowptr, p: lambda: lib.spsyrk_lookup(i64(m), i64(100), i64(p), i64(nnz), 3, rowptr, big, None, f64(1), big, i64(p), big, i64(p), None)
head = lambda: (i64(9), i64(1000), i64(18), 3, 1, None, big, big, None, None, f64(1), f64(1), big, i64(1000))
CALLS = {
    "lookup one": lookup(50, 50, None, 8), "lookup many": lookup(400_000, 400_000, None, 8), "lookup rows": lookup(50, 5000, big, 64), "lookup long": lookup(5, 5000, None, 64),
    "lookup short": lookup(50, 150, None, 8),
    "grad few": grad(500, 500, None, 1, 1), "grad sorted": grad(20_000, 20_000, None, 3, 1), "grad rows": grad(300, 20_000, big, 0, 0),
    "grad weights": lambda: lib.spsyrk_lookup_grad_weights(i64(50), i64(100), i64(8), i64(50), 1, None, big, f64(1), big, i64(8), big, i64(8), big, None),
    "distill": lambda: lib.spsyrk_distill(*head(), big, big, None, i64(0), None),
    "distill step": lambda: lib.spsyrk_distill(*head(), big, big, big, i64(1000), None),
    "distill grad": lambda: lib.spsyrk_distill_grad(*head(), big, big, i64(1000), None),
}
for name, call in CALLS.items():
    fake.fake_refuse(ctypes.c_long(-1))
    assert call() == 0, name
    launches = fake.fake_launches()
    lost = []
    for k in range(launches):
        fake.fake_refuse(ctypes.c_long(k))
        if call() != 6:
            lost.append(k)
    print(name, launches, lost, sep="|")
"""


def test_every_launch_that_fails_is_reported(tmp_path):
    from paper_2608_09713_b200 import build
    (tmp_path / "fake.cpp").write_text(launches.RUNTIME)
    fake = str(tmp_path / "libfake.so")
    subprocess.check_call(["g++", "-std=c++17", "-O1", "-w", "-shared", "-fPIC", "-o", fake, str(tmp_path / "fake.cpp")])
    out = subprocess.run([sys.executable, "-c", CALLS, fake, build.build_cuda()], env=dict(os.environ, LD_PRELOAD=fake), capture_output=True, text=True, timeout=600)
    assert out.returncode == 0, out.stdout[-2000:] + out.stderr[-2000:]
    lines = [line.split("|") for line in out.stdout.splitlines()]
    assert len(lines) == 12
    for name, count, lost in lines:
        assert int(count) > 0, name
        assert lost == "[]", f"{name}: launches {lost} of {count} failed unnoticed"
