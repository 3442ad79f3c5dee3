"""The package imports, and makes plans on the CPU, with a torch that has no GPU support."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2609_19242_amd as bd
p = bd.packed_plan([5, 3], heads=4, kv_heads=2, head_dim=64, dtype=torch.bfloat16, device="cpu")
try:
    bd.packed_fwd(p, *(torch.zeros(8, h, 64, dtype=torch.bfloat16) for h in (4, 2, 2)))
except ValueError as e:
    print("refused:", e)
"""


def test_without_gpu_support():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "refused: the tensors must be on a GPU" in r.stdout
