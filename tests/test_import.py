"""The binding loads with a torch that lacks the 4-bit types (CPU only)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import torch
for name in ("float4_e2m1fn_x2", "float8_e8m0fnu"):
    if hasattr(torch, name):
        delattr(torch, name)
from paper_2609_28870_amd import pc
assert sorted(pc._DTYPES.values()) == [0, 1, 2]
assert len(pc.rope_frequencies(8)) == 4
x = torch.zeros((2, 1, 16, 16), dtype=torch.uint8)
try:
    pc.PagedCache(x, x)
except pc.PcError as e:
    print(e)
"""


def test_a_torch_without_4_bit_types():
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr
    assert "expected two tensors" in r.stdout
