"""Gradients of weights over so many rows that one sum on the tensor cores would come out too small.

A tensor core adds 16 products and the sum so far at a time, cuts each off two bits behind the 24 of a sum and then the
result to 24 bits: 16 times an eighth and a half, 2.5 units of the sum's last place on average, each less than 2^-23 of
the sum.  With terms of one sign the sum so far is half of the last one on average.  One sum takes 65,536 rows at most,
4,096 additions, however many rows there are; those sums are added in fp32."""

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

CUT = 2.5 * 4096 / 2 * 2.0 ** -23    # 6.1e-4


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    assert torch.cuda.is_available()
    return m


def positive(n, width, g, spread=False):
    """Numbers from 1/2 to 3/2, with a gain from 1 to 2 for each column on request: results anywhere between two powers of 2."""
    t = 0.5 + torch.rand((n, width), generator=g, device="cuda")
    if spread:
        t *= 1 + torch.rand(width, generator=g, device="cuda")
    m, _ = ref.rows(n, width, 0, "cuda")
    m.copy_(t)
    return m


def long_product(d, x):
    return sum(d[i:i + 131072].double().T @ x[i:i + 131072].double() for i in range(0, x.shape[0], 131072))


def check(got, want, what):
    """Each element within a rounding to bf16 of what the sums may lose, and their mean, in which the roundings (uniform in
    2^-8 at most, four standard deviations) go away.  There are as many roundings as columns: a column's elements are sums
    of M numbers that spread by 0.4 or less around 1, times the column's gain, so that they are within 0.4 M^-1/2 of one
    another (2.3e-4 with 3,000,000 rows), less than the step of 2^-8 or more that they are rounded to, and most of them
    are rounded alike."""
    off = (got.double() - want) / want
    print(what, "mean", float(off.mean()), "most", float(off.abs().max()))
    assert float(off.abs().max()) <= CUT + ref.HALF, what
    assert abs(float(off.mean())) <= CUT + 4 * ref.HALF / (3 * off.shape[1]) ** 0.5, what


@pytest.mark.parametrize("M,N,K", [(65536, 64, 264), (65537, 70, 66), (1000003, 70, 265), (3000000, 64, 520)])
def test_weight_gradients_of_many_rows(wz, M, N, K):
    g = torch.Generator(device="cuda").manual_seed(M)
    x, dy, w = positive(M, K, g, True), positive(M, N, g), positive(N, K, g)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    workspace = torch.empty(wz.wz_linear_backward_workspace_size(M, K, N), dtype=torch.uint8, device="cuda")
    dx, dw, _ = wz.wz_linear_backward(dy, x, w, workspace=workspace, device_status=status)
    check(dw, long_product(dy, x), "dw")
    assert torch.equal(wz.wz_linear_backward(dy, x, w, need_x=False)[1], dw)
    del workspace
    gate, up = positive(M, N, g), positive(M, N, g)
    (dg, _), (du, _) = ref.gated_delta(dy, x, w, w, None, None, gate, up, "silu")
    _, dw_gate, dw_up, _, _ = wz.wz_gated_backward(dy, x, w, w, gate=gate, up=up, need_x=False, device_status=status)
    check(dw_gate, long_product(dg, x), "dw_gate")
    check(dw_up, long_product(du, x), "dw_up")
    assert int(status) == 0


def test_as_many_products_as_there_are_shares(wz):
    """Many tiles, of which each has several shares of its rows."""
    M, N, K = 150000, 1100, 900
    g = torch.Generator(device="cuda").manual_seed(1)
    x, dy, w = positive(M, K, g, True), positive(M, N, g), positive(N, K, g)
    dx, dw, _ = wz.wz_linear_backward(dy, x, w)
    check(dw, long_product(dy, x), "dw")
    want = dy.double() @ w.double()
    assert float(((dx.double() - want) / want).abs().max()) <= ref.HALF + 2.0 ** -14   # 1,100 terms
