"""The binding can be imported where torch was built without CUDA, and refuses what it is given there."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2608_09713_b200 import binding as B
try:
    B.spsyrk_lookup(torch.zeros(4, dtype=torch.int32), torch.zeros((9, 8)))
except ValueError as e:
    print(e)
"""


def test_import_without_cuda_in_torch():
    from paper_2608_09713_b200 import build
    build.build_cuda()
    run = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=600)
    assert run.returncode == 0, run.stderr[-2000:]
    assert "must be CUDA tensors" in run.stdout
