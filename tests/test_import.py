"""The package can be imported, and its host-only calls made, with a torch that
has no GPU support."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_getCurrent")]:
    delattr(torch._C, name)
import paper_2607_22866_amd as p
try:
    p.route(torch.zeros(2, 4), 1)
except ValueError as e:
    assert "CUDA tensor" in str(e)
    print("refused")
"""


def test_import_without_gpu_support():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    assert r.stdout.strip() == "refused"
