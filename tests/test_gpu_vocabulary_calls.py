"""How the lookups and the distillation are called: workspaces of the caller's own, and tensors that a graph of
torch's autograd has kept."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    from paper_2608_09713_b200 import binding
    return binding


def test_workspaces(B):
    """One of the size that is asked for is taken; a smaller one, an empty one among them, is an error and not a call that does nothing."""
    ids = torch.arange(4, dtype=torch.int32, device="cuda")
    dy = torch.ones((4, 8), device="cuda")
    expected = torch.zeros((9, 8), device="cuda")
    expected[:4] = 1
    size = B.spsyrk_lookup_grad_workspace_bytes(4, 9, 8, 4, torch.float32)
    room = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert torch.equal(B.spsyrk_lookup_grad(ids, dy, 9, workspace=room), expected)
    for bytes in (size - 1, 1, 0):
        with pytest.raises(B.SpsyrkError) as refused:
            B.spsyrk_lookup_grad(ids, dy, 9, workspace=room[:bytes])
        assert refused.value.status == 3


def test_what_is_written_into_counts_as_changed(B):
    """A backward pass that has kept a tensor before a call wrote into it raises an error; results have no graph."""
    ids = torch.arange(4, dtype=torch.int32, device="cuda")
    pairs, z = ids.view(4, 1), torch.zeros((4, 1), device="cuda")
    fresh = lambda rows, cols=8: torch.randn((rows, cols), device="cuda", requires_grad=True) * 2.0
    e, dy = torch.ones((9, 8), device="cuda"), torch.ones((4, 8), device="cuda")
    lse = torch.zeros(4, device="cuda")
    calls = [(fresh(4), lambda t: B.spsyrk_lookup(ids, e, y=t)), (fresh(9), lambda t: B.spsyrk_lookup_grad(ids, dy, 9, de=t)),
             (fresh(9), lambda t: B.spsyrk_lookup_grad(ids, dy, 9, de=t, accumulate=True)),
             (fresh(4, 1), lambda t: B.spsyrk_lookup_grad_weights(pairs, e, dy, dw=t)),
             (fresh(4), lambda t: B.spsyrk_distill(t, pairs, z, grad=t)[2]), (fresh(4), lambda t: B.spsyrk_distill_grad(t, lse, pairs, z, grad=t))]
    for kept, call in calls:
        out = (kept * kept).sum()
        assert call(kept) is kept
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            out.backward()
    e = e.requires_grad_()
    assert not B.spsyrk_lookup(ids, e).requires_grad
    out = (e * e).sum()
    B.spsyrk_lookup(ids, e)  # reads only
    out.backward()
    with torch.inference_mode():
        assert torch.equal(B.spsyrk_lookup(ids, e, y=torch.empty((4, 8), device="cuda")), e[:4])
