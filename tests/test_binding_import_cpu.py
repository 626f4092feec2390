"""The binding on a torch without CUDA (HIP) support: it can be imported, and answers
what needs no device."""

import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda_")]:
    delattr(torch._C, name)
from paper_2506_20194_amd import duo, serve
assert duo.kv_page_bytes(16, 2, 64, "int8") == 2 * 16 * 2 * (64 + 4)
x = torch.zeros((3, 64), dtype=torch.bfloat16)
try:
    duo.duo_rope_at(x, 1, 64, torch.zeros(3, dtype=torch.int32))
except ValueError as e:
    assert "device" in str(e)
else:
    raise AssertionError("a host tensor was taken")
print("fine")
"""


def test_import_without_cuda(duo_lib):
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stdout + r.stderr
