"""The binding on a torch that was built without CUDA (no GPU needed)."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CODE = """
import sys
sys.path.insert(0, {root!r})
import torch
for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):   # such a build has neither
    if hasattr(torch._C, name):
        delattr(torch._C, name)
from paper_2603_06619_b200 import nat
t, i = torch.zeros(4, 64), torch.zeros(4, dtype=torch.int32)
p = nat.embed_params(4, 64, torch.float32)
assert nat.nat_embed_workspace_bytes(p, 4) > 0
calls = [lambda: nat.nat_embed_fwd(p, t, i, None, None, 4, t),
         lambda: nat.nat_ckpt8_store(t, None, 4, torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 1)),
         lambda: nat.nat_experts_fwd(nat.experts_params(1, 64, 64, torch.float32), i, 4, t, t.view(1, 4, 64), t, t)]
for call in calls:
    try:
        call()
    except nat.NatError as e:
        assert "not on the current CUDA device" in str(e), e
    else:
        raise AssertionError("not refused")
print("refused")
"""


def test_import_sizes_and_refusals():
    r = subprocess.run([sys.executable, "-c", CODE.format(root=ROOT)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "refused" in r.stdout, r.stdout + r.stderr
