"""The binding imported before torch: both share one HIP runtime, and the library's calls run on torch's tensors."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

CODE = """
from paper_2408_10188_amd import binding as B, paged
import sys
assert "torch" not in sys.modules
import torch
x = torch.randn(3, 2, 128, device="cuda:0")
y, pos = torch.empty_like(x), torch.zeros(1, 3, dtype=torch.int32, device="cuda:0")
B.mmsp_rotary_apply(B.mmsp_rotary_plan(128, 1e6, [64]), 3, pos, 3, [paged.heads_of(x)], [paged.heads_of(y)])
torch.cuda.synchronize()
print(torch.equal(x, y), len({line.split()[-1] for line in open("/proc/self/maps") if "libamdhip64" in line}))
"""


def test_the_binding_before_torch():
    run = subprocess.run([sys.executable, "-c", CODE], cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))), check=True, capture_output=True, text=True, timeout=100)
    assert run.stdout.split() == ["True", "1"]
