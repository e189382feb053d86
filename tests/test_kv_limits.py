"""Sizes at the ends of what the decoder cache's entry points take, on the host: no call reaches the device."""

import ctypes as C
import os
import subprocess
import sys

import pytest

from test_kv_abi import append_args, attend_args, wz  # noqa: F401

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


@pytest.mark.parametrize("T,max_new,Hq,heads", [
    (1 << 30, 0, 28, 4), (1 << 30, 1 << 29, 16, 4), ((1 << 31) - 1, 0, 1, 1), (1 << 27, 0, 16, 1),
    (1 << 16, 0, 65536, 1),
])
def test_attend_refuses_rows_past_31_bits(wz, T, max_new, Hq, heads):  # noqa: F811
    """Rows of a sequence and KV head: max_new tokens of Hq / heads heads."""
    a = attend_args(wz, T=T, max_new=max_new, Hq=Hq, q_stride=Hq * 128, out_stride=Hq * 128, **{"cache.heads": heads})
    assert wz._lib.wz_attend(C.byref(a)) == -2
