"""Sizes at the ends of what the decoder cache's entry points take, on the host: no call reaches the device."""

import ctypes as C

from test_kv_abi import append_args, wz  # noqa: F401


def test_append_of_no_tokens_with_queries(wz):  # noqa: F811
    """An empty tensor has no address: a call without tokens still has its query heads."""
    a = append_args(wz, T=0, k=None, v=None, q=None, q_out=None)
    assert a.Hq == 28 and wz._lib.wz_kv_append(C.byref(a)) == 0
    assert wz._lib.wz_kv_append(C.byref(append_args(wz, T=0, q=None, q_out=None, Hq=27))) == -1
