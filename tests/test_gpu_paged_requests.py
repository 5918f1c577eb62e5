"""The plan of a step for numbers of requests at which its kernels need more shared memory than a launch has by itself, each in a process
of its own: what an earlier call has asked for would hide that one does not."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import sys
import torch
from paper_1712_01084_b200 import binding as pb
requests, rows = int(sys.argv[1]), int(sys.argv[2])
n = lambda x: torch.full((requests,), x, dtype=torch.int32, device="cuda")
table = torch.full((requests, 2), -1, dtype=torch.int32, device="cuda")
free = torch.arange(requests, dtype=torch.int32, device="cuda")
taken = torch.zeros(1, dtype=torch.int32, device="cuda")
p = pb.pp_paged_plan(n(0), n(1), table, free, taken, 4, rows=rows)
want = torch.arange(rows, device="cuda") * 4
want[requests:] = -1
assert torch.equal(p.slots, want) and p.taken.tolist() == [requests] and bool((p.lengths == 1).all())
assert torch.equal(table[:, 0], free)
print("fine")
"""


@pytest.mark.gpu
@pytest.mark.parametrize("requests", [4053, 4054, 4085, 4086, 4090, 4095, 4096, 8192])
@pytest.mark.parametrize("rows", [100, 8200, 100000])        # a row to a thread of one CTA, of several, four rows to a thread
def test_plan_of_many_requests_in_a_fresh_process(requests, rows):
    r = subprocess.run([sys.executable, "-c", PROGRAM, str(requests), str(rows)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "fine" in r.stdout, r.stderr[-500:]
