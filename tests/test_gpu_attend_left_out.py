"""Sequences with more tokens than max_new, over items of several pieces: a token's rows are right or left alone."""

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


@pytest.mark.parametrize("G,max_new,n", [(1, 1, 3), (7, 1, 2), (3, 5, 6), (5, 1, 4), (16, 1, 2), (4, 8, 12)])
@pytest.mark.parametrize("seqs", [1, 80])
def test_rows_past_max_new(wz, G, max_new, n, seqs):
    """Few and many items: both forms of the join."""
    P, D, kv = 128, 64, [4000 + 7 * b for b in range(seqs)]
    table, pages = tables(kv, P, 3)
    host = ref.Cache(pages, 1, P, D, seed=6)
    gpu = host.on_gpu(wz)
    T = n * seqs
    cu = [n * b for b in range(seqs + 1)]
    q = torch.randn((T, G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    out = torch.full((T, G, D), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((T, G), 7.0, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    workspace = torch.full((wz.wz_attend_workspace_size(T, G, D),), 0x41, dtype=torch.uint8, device="cuda")
    wz.wz_attend(q.cuda(), gpu, i32(table), i32(cu), i32(kv), max_new=max_new, out=out, lse=lse, workspace=workspace,
                 device_status=status)
    assert int(status) == wz.STATUS_CACHE
    out, lse = out.cpu().double(), lse.cpu().double()
    want, want_lse, mass, off = ref.attend(host, q, table, cu, kv, True, D ** -0.5)
    tol = 2.0 ** -9 * 1.01 * want.abs() + (2.0 ** -8 + 2.0 ** -11 + 2 * off[..., None]) * 1.05 * mass + 1e-30
    right = ((out - want).abs() <= tol).all(-1) & ((lse - want_lse).abs() <= off + 2.0 ** -20 * want_lse.abs() + 2.0 ** -19)
    alone = (out == 7).all(-1) & (lse == 7)
    assert bool((right | alone).all()), (right | alone).nonzero()[:5].tolist()
    first = torch.arange(T) % n < max_new
    assert bool(right[first].all())
