"""The binding on a torch that was built without CUDA."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2509_06980_b200 import binding as b
assert b.workspace_bytes(b.FN_NORM_BWD, 10, 0, 64, b.RLF_F32) > 0
for call in (lambda: b.rlf_norm_fwd(torch.zeros(2, 8), torch.ones(8)), lambda: b.rlf_cross_entropy_fwd_bwd(torch.zeros(2, 8), torch.zeros(2, dtype=torch.int32))):
    try:
        call()
    except ValueError as e:
        assert "CUDA" in str(e)
    else:
        raise SystemExit("a CPU tensor went through")
print("fine")
"""


def test_import_without_torchs_cuda_short_cuts():
    p = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert p.returncode == 0 and "fine" in p.stdout, p.stderr[-2000:]
