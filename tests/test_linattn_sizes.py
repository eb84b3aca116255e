"""Workspace sizes of linear attention for calls without tokens, which are no-ops:
0, at once.  Asked in a child process: a size that divides by the number of
chunks ends the process that asks."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CHILD = """
import sys
import paper_2406_02528_amd as mmf
dims = [int(x) for x in sys.argv[1:]]
print(mmf.mmf_linattn_workspace_bytes(*dims), mmf.mmf_linattn_bwd_workspace_bytes(*dims))
"""


@pytest.mark.parametrize("dims", [(2, 0, 3, 32, 48), (0, 0, 1, 16, 16), (0, 7, 3, 32, 48), (1, 0, 1, 256, 256),
                                  (2 ** 20, 0, 1, 16, 16), (0, 2 ** 31 - 1, 1, 64, 64)], ids=str)
def test_no_tokens_need_no_workspace(dims):
    r = subprocess.run([sys.executable, "-c", CHILD, *map(str, dims)], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, (r.returncode, r.stderr[-500:])
    assert r.stdout.split() == ["0", "0"]


def test_no_sequences_are_answered_without_a_search():
    """The search for the segments ends by their workgroups, of which no
    sequences have none."""
    code = """
import time
import paper_2406_02528_amd as mmf
t = time.process_time()
for _ in range(200):
    assert mmf.mmf_linattn_workspace_bytes(0, 2 ** 31 - 1, 1, 64, 64) == 0
    assert mmf.mmf_linattn_bwd_workspace_bytes(0, 2 ** 31 - 1, 1, 64, 64) == 0
print(time.process_time() - t)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-500:]
    assert float(r.stdout) < 5.0
