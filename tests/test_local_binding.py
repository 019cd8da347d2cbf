"""The local-gradient binding on the CPU: what its import needs of torch."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

WITHOUT_GPU_NAMES = """
import torch
for name in ("_cuda_getCurrentRawStream", "_cuda_getDevice"):
    if hasattr(torch._C, name):
        delattr(torch._C, name)
import paper_2507_07114_amd as ll
tokens = torch.zeros((2, 5), dtype=torch.int32)
try:
    ll.ll_embed(tokens, torch.zeros(2, 80), torch.zeros(2, 5, 8), v=10)
except ValueError as e:
    assert "on one GPU" in str(e), e
else:
    raise AssertionError("tensors on the CPU were taken")
assert ll.ll_workspace_bytes(2, 100, 10) > 0
print("ok")
"""


def test_import_with_a_torch_without_gpu_support():
    # such a torch lacks the private names that read the current stream; it has
    # no GPU tensors, so no call gets as far as them
    r = subprocess.run([sys.executable, "-c", WITHOUT_GPU_NAMES], cwd=ROOT, capture_output=True,
                       text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stderr
