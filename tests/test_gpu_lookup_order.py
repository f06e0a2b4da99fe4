"""The gradient of a lookup from an order of its entries that is not whole, as the sort leaves it after one of its waits has run out: entries of
rows that are not there add nothing and nothing is read for them, and the error word turns every sum into NaN.  The kernels behind
the sort are built by themselves and given such an order."""
import ctypes
import os
import subprocess

import pytest
import torch

pytestmark = pytest.mark.gpu
CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_09713_b200", "csrc")

SOURCE = r"""
#include "lookup_grad.cu"
namespace spsyrk { void note_launches(int) {} }
extern "C" long order_workspace(int64_t n, int64_t p, int64_t nnz) { return (long)carve(nullptr, nullptr, n, p, nnz, false, true); }
// the sums of the entries (key[e], row[e]) in the order in which they are given
extern "C" int add_in_order(int64_t m, int64_t n, int64_t p, int64_t nnz, uint32_t* key, uint32_t* row, const uint32_t* err, const float* dy, float* de, void* workspace) {
    GradWs w;
    carve(&w, workspace, n, p, nnz, false, true);
    w.key[0] = key;
    w.row[0] = row;
    const Fill none{nullptr, 0, 0, 4, 0, n};
    const int status = p % 4 == 0 ? add_typed<float, float, 4>(w, 0, err, none, m, n, p, nnz, false, 1.0, dy, p, de, p, false, nullptr)
                                  : add_typed<float, float, 1>(w, 0, err, none, m, n, p, nnz, false, 1.0, dy, p, de, p, false, nullptr);
    return status ? status : (int)cudaDeviceSynchronize();
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    from paper_2608_09713_b200 import build
    d = tmp_path_factory.mktemp("order")
    (d / "order.cu").write_text(SOURCE)
    out = str(d / "liborder.so")
    subprocess.check_call([os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc"), *build.NVCC_FLAGS, "-I", CSRC, "-shared", "-o", out, str(d / "order.cu"), "-lcudart"])
    lib = ctypes.CDLL(out)
    lib.order_workspace.restype = ctypes.c_long
    return lib


def _add(lib, m, n, p, key, row, err, dy, de):
    i64, at = ctypes.c_int64, lambda t: None if t is None else ctypes.c_void_p(t.data_ptr())
    nnz = key.numel()
    workspace = torch.full((lib.order_workspace(i64(n), i64(p), i64(nnz)),), 255, dtype=torch.uint8, device="cuda")
    torch.cuda.synchronize()
    assert lib.add_in_order(i64(m), i64(n), i64(p), i64(nnz), at(key), at(row), at(err), at(dy), at(de), at(workspace)) == 0


@pytest.mark.parametrize("p", [64, 33, 1000])
@pytest.mark.parametrize("nnz", [40, 9000])
def test_an_order_that_is_not_whole(lib, nnz, p):
    g = torch.Generator(device="cuda")
    g.manual_seed(nnz + p)
    m, n = 500, 70
    key = torch.randint(0, n + 1, (nnz,), generator=g, device="cuda").sort()[0]
    row = torch.randint(0, m, (nnz,), generator=g, device="cuda")
    dy = torch.randint(-3, 4, (m, p), generator=g, device="cuda").float()  # (whole numbers: sums are exact)
    lost = (torch.rand(nnz, generator=g, device="cuda") < 0.2) & (key >= n // 2)
    at = torch.arange(nnz, device="cuda")
    # words that were never written: rows that are not there beside keys that may be, and keys that may be of no id
    row = torch.where(lost, torch.tensor([m, 2 ** 32 - 1, 2 ** 31, 2 ** 31 - 1], device="cuda")[at % 4], row)
    key = torch.where(lost & (at % 3 == 0), 2 ** 32 - 1, key)
    expected = torch.zeros((n + 1, p), device="cuda").index_add_(0, key[~lost], dy[row[~lost]])[:n]
    words = lambda x: torch.where(x >= 2 ** 31, x - 2 ** 32, x).to(torch.int32)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    for e in (None, err):
        de = torch.zeros((n, p), device="cuda")
        _add(lib, m, n, p, words(key), words(row), e, dy, de)
        # a run beside a lost place may be cut there; the others are whole
        cut = torch.zeros(n + 1, dtype=torch.bool, device="cuda")
        for shift in (-1, 0, 1):
            cut[key[(at[lost] + shift).clamp(0, nnz - 1)].clamp(max=n)] = True
        assert int((~cut[:n]).sum()) >= n // 2 - 1
        assert torch.equal(de[~cut[:n]], expected[~cut[:n]])
    # an order that is whole, and the word set
    key, row = torch.arange(nnz, device="cuda") * n // nnz, torch.arange(nnz, device="cuda") % m
    expected = torch.zeros((n, p), device="cuda").index_add_(0, key, dy[row])
    de = torch.zeros((n, p), device="cuda")
    _add(lib, m, n, p, words(key), words(row), err, dy, de)
    assert torch.equal(de, expected)
    _add(lib, m, n, p, words(key), words(row), err.fill_(8), dy, de)
    assert de[torch.unique(key)].isnan().all()
