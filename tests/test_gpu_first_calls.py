"""A process's first calls, from several threads at once."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

FIRST_CALLS = """
import threading, torch
import paper_2304_14698_b200 as xrl
n = 8
g = [torch.randn(64, 64, device="cuda") for _ in range(n)]
start, errors, outs = threading.Barrier(n), [], [None] * n
streams = [torch.cuda.Stream() for _ in range(n)]
torch.cuda.synchronize()
def work(i):
    start.wait()
    try:
        outs[i] = xrl.xrl_orthogonalise(g[i], stream=streams[i].cuda_stream)
    except Exception as e:
        errors.append(repr(e))
threads = [threading.Thread(target=work, args=(i,)) for i in range(n)]
for t in threads: t.start()
for t in threads: t.join()
torch.cuda.synchronize()
assert not errors, errors
for i in range(n):
    assert torch.equal(outs[i], xrl.xrl_orthogonalise(g[i]))
print("alike")
"""


def test_the_first_updates_of_a_process_may_come_from_several_threads():
    for _ in range(2):
        r = subprocess.run([sys.executable, "-c", FIRST_CALLS], capture_output=True, text=True, cwd=ROOT, timeout=300)
        assert r.returncode == 0 and "alike" in r.stdout, r.stderr[-2000:]
