"""Attention whose waits give up at once (the checked build's limit): every variant ends, says so, and leaves the GPU and
the workspace fit for the next call."""

import contextlib
import ctypes as C

import pytest
import torch

import kv_reference as ref
from test_gpu_attend import compare
from test_gpu_kv_append import i32, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


@contextlib.contextmanager
def impatient(wz, ns=1):
    """The checked library, whose waits give up after ns."""
    hook = C.CDLL(wz.LIB_CHECKED_PATH).wz_check_attend_wait
    hook.argtypes, hook.restype = [C.c_uint64], None
    hook(ns)
    try:
        with wz.checked_library():
            yield
    finally:
        torch.cuda.synchronize()
        hook(0)


VARIANTS = [
    # page, heads, heads of a group, D, new tokens, kv_len
    (64, 4, 1, 64, 1, [5000] * 8),         # one row an item, several items to a CTA
    (32, 2, 7, 128, 1, [20000, 300]),      # eight rows, pieces
    (64, 2, 8, 128, 2, [6000] * 5),        # sixteen rows
    (64, 2, 4, 128, 1, [400, 0, 512]),     # whole items
    (64, 2, 4, 128, 30, [3000, 100]),      # both row tiles hold the same rows
    (64, 1, 2, 96, 700, [5000]),           # row tiles with splits
    (16, 8, 8, 128, 200, [900] * 6),       # row tiles without
]


@pytest.mark.parametrize("case", VARIANTS, ids=[str(i) for i in range(len(VARIANTS))])
def test_calls_end_and_the_next_is_right(wz, case):
    P, heads, G, D, n, kv = case
    table, pages = tables(kv, P, 3)
    host = ref.Cache(pages, heads, P, D, seed=6)
    gpu = host.on_gpu(wz)
    T, Hq = n * len(kv), heads * G
    q = torch.randn((T, Hq, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    cu = [n * b for b in range(len(kv) + 1)]
    args = (q.cuda(), gpu, i32(table), i32(cu), i32(kv))
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    workspace = torch.zeros(wz.wz_attend_workspace_size(T, Hq, D), dtype=torch.uint8, device="cuda")
    with impatient(wz):
        for _ in range(3):
            wz.wz_attend(*args, max_new=n, workspace=workspace, device_status=status)
    assert int(status) & wz.STATUS_WAIT_TIMEOUT
    if T * Hq * max(kv) > 1 << 23:      # what the reference takes too long for: against the ordinary build
        want = wz.wz_attend(*args, max_new=n)
        assert torch.equal(wz.wz_attend(*args, max_new=n, workspace=workspace), want) and bool(torch.isfinite(want).all())
        return
    lse = torch.empty((T, Hq), device="cuda")
    out = wz.wz_attend(*args, max_new=n, workspace=workspace, lse=lse)
    assert bool(torch.isfinite(out).all())
    compare(out, lse, host, q, table, cu, kv, True, D ** -0.5)


@pytest.mark.parametrize("first,pieces", [(2 ** 31 - 1, 2), (2 ** 31 - 1, 2 ** 31 - 1), (-1, 5), (5, -1), (0, 2 ** 31 - 1),
                                          (400, 2 ** 30), (-2 ** 31, -2 ** 31)])
def test_pieces_that_nobody_wrote(wz, first, pieces):
    """Items whose CTAs gave up before they wrote where their pieces lie: the join finds what the workspace held."""
    P, heads, D, kv = 32, 2, 64, [5000] * 40
    table, pages = tables(kv, P, 3)
    gpu = ref.Cache(pages, heads, P, D, seed=6).on_gpu(wz)
    q = torch.randn((40, 4, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    args = (q, gpu, i32(table), i32(list(range(41))), i32(kv))
    want = wz.wz_attend(*args, max_new=1).clone()
    workspace = torch.empty(wz.wz_attend_workspace_size(40, 4, D) // 8 * 8, dtype=torch.uint8, device="cuda")
    workspace.view(torch.int32).view(-1, 2)[:] = i32([first, pieces])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with impatient(wz):
        wz.wz_attend(*args, max_new=1, workspace=workspace, device_status=status)
    assert int(status) == wz.STATUS_WAIT_TIMEOUT
    assert torch.equal(wz.wz_attend(*args, max_new=1, workspace=workspace), want)
