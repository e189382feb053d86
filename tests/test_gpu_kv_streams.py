"""Outputs that the binding allocates for a call on a given stream belong to that stream."""

import pytest
import torch

import kv_reference as ref
from test_gpu_kv_append import i32, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


def test_outputs_do_not_come_from_another_streams_memory(wz):
    """Memory freed on the current stream may still be in use there, so a call on another stream must not get it."""
    T, heads, Hq, D, P = 64, 2, 8, 64, 64
    table, pages = tables([T], P, 3)
    gpu = ref.Cache(pages, heads, P, D, seed=6).on_gpu(wz)
    qkv = torch.randn((T, Hq + 2 * heads, D), device="cuda").bfloat16()
    t, cu, start, kv = i32(table), i32([0, T]), i32([0]), i32([T])
    rotation = wz.rotation_table(T, D)
    q = qkv[:, :Hq]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    calls = (lambda: wz.wz_kv_append(qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], gpu, t, cu, start, q=q, rotation=rotation,
                                     stream=side),
             lambda: wz.wz_attend(q, gpu, t, cu, kv, stream=side))
    for call in calls:
        freed = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        address = freed.data_ptr()
        del freed
        got = call()
        assert got.data_ptr() != address
        again = torch.empty((T, Hq, D), dtype=torch.bfloat16, device="cuda")
        assert again.data_ptr() == address      # the block was there to be taken
        side.synchronize()
        del got, again
