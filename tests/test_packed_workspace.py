"""The context's own workspace of the attention over the 4-bit cache: a refused call leaves none behind.  In processes of their own, as no device is
needed for what is refused."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SCRIPT = """
import ctypes, sys
import torch
from paper_2408_15562_b200 import binding
binding._stream = lambda s: 0
bf, i32, u8 = torch.bfloat16, torch.int32, torch.uint8
ctx = binding.Context.__new__(binding.Context)
ctx._h, ctx._sizes, ctx._workspace, ctx.cfg = ctypes.c_void_p(), (8, 2, 1, 4), None, binding.FspadConfig(8, 2, 128, 4, 16, 1, 512, 1, 0.0)
def fake(*shape, dtype=bf, at="cuda:0"):
    from torch._subclasses.fake_tensor import FakeTensorMode
    with FakeTensorMode(): return torch.empty(shape, dtype=dtype, device=at)
a = dict(q=fake(1, 4, 8, 128), codes=fake(1, 2, 5, 2, 128, 64, dtype=u8), scales=fake(1, 2, 5, 2, 128, 8, dtype=u8), block_table=fake(1, 6, dtype=i32),
         tree_k=fake(1, 2, 4, 128), tree_v=fake(1, 2, 4, 128), parent=fake(1, 4, dtype=i32), prefix_len=fake(1, dtype=i32), out=fake(1, 4, 8, 128))
bad = dict(q=torch.zeros((1, 4, 8, 128), dtype=bf), q_list=[1.0], tree_k=torch.zeros((1, 2, 4, 128), dtype=bf), parent=fake(1, 5, dtype=i32), context=None)
what = sys.argv[1]
if what != "context": a[what.split("_list")[0]] = bad[what]
try:
    ctx.tree_attn_packed(**a)
    print("returned")
except Exception as e:
    print(type(e).__name__, str(e).splitlines()[0] if str(e) else "", "| kept:", ctx._workspace is not None)
"""


@pytest.mark.parametrize("what,kind", [("q", "ValueError"), ("q_list", "TypeError"), ("tree_k", "ValueError"), ("parent", "ValueError"), ("context", "FspadError")])
def test_a_refused_call_leaves_no_workspace_behind(what, kind):
    r = subprocess.run([sys.executable, "-c", SCRIPT, what], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    assert r.stdout.startswith(kind) and r.stdout.rstrip().endswith("kept: False"), r.stdout
