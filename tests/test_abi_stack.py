"""Lists of matrices from threads with small stacks: the host side of a call keeps
what grows with the longest list off the caller's stack (each runs in a process of
its own, which an overflow would end)."""

import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
PROGRAM = """
import ctypes, sys, threading
import paper_1911_07384_amd as F
count = int(sys.argv[1])
F.lib()
descs = F.muon_descs([(64 + i % 3, 1100) for i in range(count)])
far = lambda base: (ctypes.c_void_p * count)(*[base + (1 << 20) * i for i in range(count)])
a, b = far(1 << 40), far(2 << 40)
def calls():
    need = F.fp16_muon_workspace_bytes(descs)
    assert need > 0 and F.fp16_muon_kernels(descs)
    # (the workspace over a matrix: refused after everything else has been looked at)
    assert F.lib().fp16_orthogonalize(count, descs, a, b, 5, None, 1, b[count - 1], need, None) == 5
    assert F.lib().fp16_muon_step(count, descs, a, b, far(3 << 40), 0.1, 0.9, 0.0, 1, 5, None, 1,
                                  a[0], need, None) == 5
    print("done")
threading.stack_size(128 << 10)
t = threading.Thread(target=calls)
t.start()
t.join()
"""


@pytest.mark.parametrize("count", [1, 1024])
def test_a_stack_of_128_kib(count):
    r = subprocess.run([sys.executable, "-c", PROGRAM, str(count)], cwd=ROOT, capture_output=True,
                       text=True, timeout=120)
    assert r.returncode == 0 and r.stdout == "done\n", (r.returncode, r.stderr[-500:])
