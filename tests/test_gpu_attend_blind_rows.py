"""Rows that see no slot, of queries with infinities and NaN: 0 and -infinity, as for any other query."""

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


@pytest.mark.parametrize("n,kv,G", [
    (4, 1, 2),         # few rows
    (40, 10, 2),       # one tile of rows, held by both
    (150, 37, 1),      # two tiles
    (300, 130, 1),     # a CTA whose rows all see nothing beside one whose rows do
])
def test_nonfinite_queries_that_see_nothing(wz, n, kv, G):
    P, D = 32, 64
    table, pages = tables([kv], P, 3)
    gpu = ref.Cache(pages, 1, P, D, seed=6).on_gpu(wz)
    q = torch.randn((n, G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    args = (i32(table), i32([0, n]), i32([kv]))

    def call(x):
        lse = torch.full((n, G), 7.0, device="cuda")
        return wz.wz_attend(x.cuda(), gpu, *args, lse=lse).cpu().float(), lse.cpu()

    want, want_lse = call(q)
    bad = q.clone()
    blind = n - kv                       # the first tokens, which no slot is left for
    bad[0, 0, 7], bad[blind - 1, G - 1, 3] = float("nan"), float("inf")
    bad[blind // 2, 0, 5] = float("-inf")
    bad[n - 1, 0, 1] = float("nan")      # this one sees all slots
    got, lse = call(bad)
    assert bool((got[:blind] == 0).all()) and bool(torch.isneginf(lse[:blind]).all())
    assert bool(torch.isnan(got[n - 1, 0]).all()) and bool(torch.isnan(lse[n - 1, 0]))
    same = torch.ones((n, G), dtype=torch.bool)
    same[n - 1, 0] = False
    assert torch.equal(got[same], want[same]) and torch.equal(lse[same], want_lse[same])
