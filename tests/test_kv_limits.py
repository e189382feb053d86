"""Sizes at the ends of what the decoder cache's entry points take, on the host: no call reaches the device."""

import ctypes as C
import os
import subprocess
import sys

import pytest

from test_kv_abi import append_args, wz  # noqa: F401

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_append_of_no_tokens_with_queries(wz):  # noqa: F811
    """An empty tensor has no address: a call without tokens still has its query heads."""
    a = append_args(wz, T=0, k=None, v=None, q=None, q_out=None)
    assert a.Hq == 28 and wz._lib.wz_kv_append(C.byref(a)) == 0
    assert wz._lib.wz_kv_append(C.byref(append_args(wz, T=0, q=None, q_out=None, Hq=27))) == -1


HEADS = """
import ctypes as C, sys
sys.path[:0] = [{root!r}, {tests!r}]
import paper_2607_23265_gb300.wavezip as wz
from test_kv_abi import append_args
a = append_args(wz, Hq={Hq}, q_stride={Hq} * 128, q_out_stride={Hq} * 128)
print("returned", wz._lib.wz_kv_append(C.byref(a)))
"""


@pytest.mark.parametrize("Hq", [65540, 1 << 28, 1 << 29, (1 << 31) - 4])
def test_append_refuses_more_heads_than_attention_takes(wz, Hq):  # noqa: F811
    """In a process of its own: an arithmetic fault would end it."""
    program = HEADS.format(root=ROOT, tests=os.path.join(ROOT, "tests"), Hq=Hq)
    r = subprocess.run([sys.executable, "-c", program], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["returned", "-2"], (r.returncode, r.stdout, r.stderr[-500:])
