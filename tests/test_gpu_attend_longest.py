"""Lengths at the end of 31 bits."""

import pytest
import torch

from test_gpu_kv_append import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


@pytest.mark.parametrize("kv,cut", [(2 ** 31 - 257, False), (2 ** 31 - 256, True), (2 ** 31 - 1, True)])
def test_slots_that_are_not_read_are_reported(wz, kv, cut):
    """A table whose 2^24 entries name one page: the sequence's slots past 2^31 - 257 are left out and reported."""
    P, D = 128, 16
    cache = wz.KvCache.empty(1, 1, P, D)
    cache.v.copy_(torch.ones((1, 1, P, D), device="cuda"))
    table = torch.zeros((1, 1 << 24), dtype=torch.int32, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.ones((1, 1, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((1, 1), device="cuda")
    out = wz.wz_attend(q, cache, table, i32([0, 1]), i32([kv]), max_new=1, lse=lse, device_status=status)
    assert int(status) == (wz.STATUS_CACHE if cut else 0)
    assert bool((out == 1).all())
    assert abs(float(lse) - 31 * 0.6931471805599453) < 1e-5
