"""Refusals of several host threads at once: each thread reads its own.  No GPU needed."""
import os
import subprocess
import sys

PROGRAM = """
import threading
import paper_2302_01318_b200 as sps

L = sps.lib()
gate, wrong = threading.Barrier(8), []


def run(i):
    gate.wait()
    for _ in range(20000):
        if i % 2:
            code, text = L.sps_paged_pool_workspace_bytes(0), b"n_pages must be 1 .. 2^20"
        else:
            code, text = L.sps_beam_select_workspace_bytes(1, 0, 8), b"beams: B must be 0 .. 8192, W 1 .. 128, V 1 .. 2^24"
        if code != -1 or L.sps_last_error(None) != text:
            wrong.append(code)


threads = [threading.Thread(target=run, args=(i,)) for i in range(8)]
for t in threads:
    t.start()
for t in threads:
    t.join()
assert not wrong, len(wrong)
"""


def test_each_thread_reads_its_own_refusal():
    """In a process of its own: texts written at once could end it."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", PROGRAM], cwd=root, env={**os.environ, "PYTHONPATH": root}, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]
