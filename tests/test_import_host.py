"""The package on a torch that was built without CUDA: it imports, its host-only calls work, and calls on host tensors are refused as everywhere."""
import os
import subprocess
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

CODE = """
import torch
for name in [n for n in dir(torch._C) if n.startswith("_cuda")]:
    delattr(torch._C, name)
import paper_2608_28276_b200 as P
assert P.pask_rotary_table(64, device="cpu").numel() == 32
x, ids = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(1, dtype=torch.int32)
q, kv = torch.zeros(3, 8, 128, dtype=torch.bfloat16), torch.zeros(3, 2, 128, dtype=torch.bfloat16)
cu, ws = torch.tensor([0, 3], dtype=torch.int32), torch.zeros(256, dtype=torch.uint8)
for call in (lambda: P.pask_rotary(torch.zeros(3, dtype=torch.int32), P.pask_rotary_table(64, device="cpu"), [(x, x)]),
             lambda: P.pask_prompt_attention(1, 0, ids, cu, q, kv, kv, q.clone(), None, ws)):
    try:
        call()
    except P.PaskError as e:
        assert e.status == P.ERR_INVALID_ARG
    else:
        raise AssertionError("not refused")
print("fine")
"""


def test_imports_without_cuda_in_torch():
    r = subprocess.run([sys.executable, "-c", CODE], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "fine", r.stderr
