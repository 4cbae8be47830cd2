"""Importing the binding needs public names of PyTorch only."""
import os
import subprocess
import sys

CODE = """
import torch
if hasattr(torch._C, "_cuda_getCurrentRawStream"):
    del torch._C._cuda_getCurrentRawStream
from paper_2407_00952_b200 import binding as B
try:
    B.quantize_rows(torch.zeros(4, 64, dtype=torch.float64))
except B.SplitLoraError as e:
    assert e.code == -1
else:
    raise SystemExit("not refused")
"""


def test_binding_imports_where_pytorch_lacks_its_private_names():
    """A build without CUDA, or a later one."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", CODE], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
