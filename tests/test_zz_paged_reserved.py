"""The paged operators where a reservation leaves no room for parts: nothing is split, the results are as exact.  A process of its own, because a
reservation holds until the process ends."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
HERE = os.path.dirname(os.path.abspath(__file__))

CHILD = r'''
import random
import sys
sys.path.insert(0, %r), sys.path.insert(0, %r)
import paper_2403_01136_amd as lpq
import test_gpu_paged as t
lpq.load_library()
lpq.lpq_workspace_reserve(1024)
size = lpq.lpq_workspace_bytes()
t.check_attention(*t.Paged([(5000, 1), (30, 1), (0, 1), (777, 1)], 8, 2, 128, 16, "fp16", 2).run(max_q=1), what="decode")
t.check_attention(*t.Paged([(2000, 3), (31, 4)], 10, 2, 64, 32, "bf16").run(True, max_q=4), what="two column tiles")
t.check_attention(*t.Paged([(3000, 100)], 8, 2, 128, 64, "fp16").run(max_q=100), what="chunk")
t.check_attention(*t.Paged([(900, 1), (2100, 200), (17, 1)], 8, 8, 64, 16, "bf16", 5).run(max_q=200), what="mixed")
t.check_attention(*t.packed_run([1100, 60], 2, 1, 128, "fp16", True), what="packed")
r = random.Random(1)
t.check_plan(t.plan_case(5, 300, 32, lambda r: r.choice((1, 80)), 300, 4), 32)
assert lpq.lpq_workspace_bytes() == size, "the workspace has grown"
print("RESERVED OK")
'''


def test_no_room_for_parts():
    out = subprocess.run([sys.executable, "-c", CHILD % (os.path.dirname(HERE), HERE)], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0 and "RESERVED OK" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]


CHILD_PLAN = r'''
import sys
sys.path.insert(0, %r), sys.path.insert(0, %r)
import paper_2403_01136_amd as lpq
import test_gpu_paged as t
lpq.load_library()
case = t.plan_case(5, 30, 32, lambda r: r.choice((300, 800)), 300, 4)
assert case[-1] > 10000
t.check_plan(case, 32)
assert lpq.lpq_workspace_bytes() == 0, "a plan has made a workspace"
print("PLAN OK")
'''


def test_plans_use_no_workspace():
    out = subprocess.run([sys.executable, "-c", CHILD_PLAN % (os.path.dirname(HERE), HERE)], capture_output=True, text=True, timeout=110)
    assert out.returncode == 0 and "PLAN OK" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]


CHILD_SOME = r'''
import sys
sys.path.insert(0, %r), sys.path.insert(0, %r)
import torch
import paper_2403_01136_amd as lpq
import test_gpu_paged as t
lpq.load_library()
batches = [t.Paged([(30000, 1), (3000, 64), (0, 1)], 32, 8, 128, 64, "fp16", 2), t.Paged([(2000, 1), (3000, 40)], 40, 2, 64, 16, "bf16")]
times = []
for mb in (20, 45, 600):
    lpq.lpq_workspace_reserve(mb << 20)
    size = lpq.lpq_workspace_bytes()
    assert size == mb << 20
    for p in batches:
        t.check_attention(*p.run(max_q=64), what="%%d MiB" %% mb)
    p = batches[0]
    args = (p.qkv, p.k, p.v, t.ints(p.table), t.ints(p.cu), t.ints([a + b for a, b in p.seqs]))
    best = 1e9
    for _ in range(5):
        a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
        a.record()
        lpq.lpq_paged_attention(*args, max_q=64, max_kv=30001)
        b.record()
        torch.cuda.synchronize()
        best = min(best, a.elapsed_time(b))
    times.append(best)
    assert lpq.lpq_workspace_bytes() == size, "the workspace has grown"
print("ms", times)
assert times[0] <= 8 * times[2] and times[1] <= 4 * times[2], times
print("RESERVED OK")
'''


def test_room_for_some_parts():
    """Room for the streaming kernel's parts alone, then for some of the tile kernel's too: a long decode beside a chunk is not left to one wave."""
    out = subprocess.run([sys.executable, "-c", CHILD_SOME % (os.path.dirname(HERE), HERE)], capture_output=True, text=True, timeout=110)
    print(out.stdout[-300:])
    assert out.returncode == 0 and "RESERVED OK" in out.stdout, out.stdout[-2000:] + out.stderr[-4000:]
