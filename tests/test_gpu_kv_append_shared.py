"""wz_kv_append at sizes whose shared memory ends just below 48 KiB, each as the first call of its process: the
limit that a larger call before it raised would hide a launch that the driver refuses."""

import os
import subprocess
import sys

import pytest

pytestmark = pytest.mark.gpu

TESTS = os.path.dirname(os.path.abspath(__file__))

PROGRAM = """
import sys
sys.path[:0] = [{root!r}, {tests!r}]
import paper_2607_23265_gb300.wavezip as wz
import test_gpu_kv_append as t
t.test_append(wz, {case!r})
print("appended")
"""

CASES = [
    # page, heads, Hq, D, new, start, dtype, rot, interleaved, axes: rows x (rot + axes) x 4 bytes
    (128, 2, 4, 96, [130], [0], "bf16", 96, False, 1),     # 128 x 96 x 4 = 49,152
    (128, 2, 4, 128, [96], [0], "bf16", 128, False, 1),    # 96 x 128 x 4 = 49,152
    (128, 2, 4, 96, [124], [0], "bf16", 96, False, 3),     # 124 x 99 x 4 = 49,104
    (128, 1, 2, 96, [128], [3], "f32", 96, True, 1),       # 128 x 96 x 4 = 49,152
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_first_call(case):
    import __graft_entry__
    __graft_entry__.build()
    program = PROGRAM.format(root=os.path.dirname(TESTS), tests=TESTS, case=case)
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "appended" in r.stdout, r.stderr[-2000:]
