"""Workspace sizes of linear attention.  Calls without tokens are no-ops and need
none, which is told at once (asked in a child process: a size that divides by the
number of chunks ends the process that asks).  A buffer for several lengths is the
largest of their sizes."""
import os
import subprocess
import sys

import pytest

from record import call, record

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


@pytest.mark.parametrize("dims", [(1, 16, 128, 128), (4, 2, 64, 96), (3, 8, 256, 16)], ids=str)
def test_one_buffer_serves_all_lengths_when_it_is_the_largest(dims):
    """Sizes go by the shape and may fall as T grows: the largest of them, not
    that of the longest sequence, serves every length, and less than a length's
    own size is refused for it."""
    import paper_2406_02528_amd as mmf
    B, H, dk, dv = dims
    lengths = [1, 40, 200, 500, 1000, 2048, 3073, 8192]
    P = 0x100000000
    for kind, size in (("fwd", mmf.mmf_linattn_workspace_bytes), ("bwd", mmf.mmf_linattn_bwd_workspace_bytes)):
        sizes = [size(B, T, H, dk, dv) for T in lengths]

        def run(T, n):
            shape = (B, T, H, dk, dv)
            if kind == "fwd":
                return call("mmf_linattn_fwd", P, 1, P, P, P, P, *shape, P, n, None)
            return call("mmf_linattn_bwd", P, 1, P, P, P, 1, P, P, P, *shape, P, n, None)

        rs = record([run(T, max(sizes)) for T in lengths] + [run(T, n - 1) for T, n in zip(lengths, sizes) if n])
        assert [r["status"] for r in rs] == [0] * len(lengths) + [6] * sum(n > 0 for n in sizes)
        assert all(r["allocs"] == 0 for r in rs)
