"""How the lookups and the distillation are called: workspaces of the caller's own."""
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
