"""Attention over 4-bit cells where a reservation leaves no room for parts, or for some: nothing or less is split, the results are as exact.  A process of its own, because a
reservation holds until the process ends."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = r'''
import sys
sys.path.insert(0, %r), sys.path.insert(0, %r)
import paper_2403_01136_amd as lpq
import test_gpu_cells as t
lpq.load_library()
for mb in (0, 20, 45, 600):
    lpq.lpq_workspace_reserve(mb << 20 or 1024)
    size = lpq.lpq_workspace_bytes()
    t.check_attention(*t.Cells([(5000, 1), (30, 1), (0, 1), (777, 1)], 8, 2, 128, 16, "fp16", 2).run(max_q=1), what="decode")
    t.check_attention(*t.Cells([(2000, 3), (31, 4)], 10, 2, 64, 32, "bf16").run(True, max_q=4), what="two column tiles")
    t.check_attention(*t.Cells([(3000, 100)], 8, 2, 128, 64, "fp16").run(max_q=100), what="chunk")
    t.check_attention(*t.Cells([(900, 1), (2100, 200), (17, 1)], 8, 8, 64, 16, "bf16", 5).run(max_q=200), what="mixed")
    t.check_attention(*t.Cells([(30000, 1), (3000, 64), (0, 1)], 32, 8, 128, 64, "fp16", 2).run(max_q=64), what="long beside a chunk")
    assert lpq.lpq_workspace_bytes() == size, "the workspace has grown"
    print("MiB", mb, flush=True)
print("RESERVED OK")
'''

CHILD_NONE = r'''
import sys
sys.path.insert(0, %r), sys.path.insert(0, %r)
import torch
import paper_2403_01136_amd as lpq
import test_gpu_cells as t
lpq.load_library()
p = t.Cells([(30, 50)], 8, 2, 128, 16, "fp16")
slots = t.ints(list(range(50)))
lpq.lpq_qk_norm_rotary(p.qkv, slots, 8, 2, cos_sin=t.rotary_table(50, 64))
lpq.lpq_paged_append4(p.qkv, p.k, p.v, slots)
lpq.lpq_paged_load4(p.k, p.v, slots, p.qkv)
torch.cuda.synchronize()
assert lpq.lpq_workspace_bytes() == 0, "a workspace was made"
print("NONE OK")
'''


@pytest.mark.parametrize("child,word", [(CHILD, "RESERVED OK"), (CHILD_NONE, "NONE OK")], ids=["little room", "no workspace"])
def test_workspace(child, word):
    out = subprocess.run([sys.executable, "-c", child % (os.path.dirname(HERE), HERE)], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0 and word in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]
