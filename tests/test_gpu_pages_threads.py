"""Host threads, each with a pool, a table and a stream of its own, whose first calls meet."""
import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

PROGRAM = """
import threading
import torch
import paper_2302_01318_b200 as sps

torch.zeros(1, device="cuda")
i32 = dict(dtype=torch.int32, device="cuda")
work = []
for n in (24576, 6000, 12000, 5000, 20000, 7000):
    pool, table = sps.PagePool(torch.zeros(n, **i32), 8), sps.PageTable(torch.zeros(2, n, **i32), torch.zeros(2, **i32), torch.zeros(2, **i32))
    moves, ws = sps.PageMoves(torch.zeros(2, 3, **i32), torch.zeros(1, **i32)), torch.zeros(sps.sps_paged_pool_workspace_bytes(n), dtype=torch.uint8, device="cuda")
    work.append((pool, table, torch.tensor([8 * n - 16, 9], **i32), moves, ws, torch.cuda.Stream().cuda_stream))
torch.cuda.synchronize()
gate, failed = threading.Barrier(len(work)), []


def run(pool, table, want, moves, ws, stream):
    gate.wait()
    try:
        for _ in range(20):
            sps.sps_paged_reserve(pool, table, want, moves, ws, stream=stream)
    except Exception as e:
        failed.append(e)


threads = [threading.Thread(target=run, args=w) for w in work]
for t in threads:
    t.start()
for t in threads:
    t.join()
torch.cuda.synchronize()
assert not failed, failed
for pool, table, *_ in work:
    n = pool.refs.numel()
    assert table.held.tolist() == [n - 2, 2] and bool((pool.refs == 1).all()) and int(pool.status) == 0
"""


def test_pools_of_unlike_sizes_from_threads_of_their_own():
    """Every pool asks for another amount of shared memory; run in a process of its own, whose first calls these are."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, env={**os.environ, "PYTHONPATH": root}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
