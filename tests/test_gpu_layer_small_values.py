"""Activations far below 0, where the logistic function is below the least normal number and its product with x is not.

The products are zeros and the bias is the argument, exactly: what a value is off comes from the activation alone.  It is
bounded as in layer_reference, 2^-15 relative and 2^-126, and a rounding to bf16."""

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

FAR = {"silu": (-94.0, -80.0), "gelu_tanh": (-10.3, -9.3), "gelu": (-13.4, -12.0)}


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture
def forced(wz):
    with wz.checked_library():
        yield wz._lib.wz_check_mm_plan
        wz._lib.wz_check_mm_plan(0, 1, 64)


@pytest.mark.parametrize("plan", [(0, 1, 64), (1, 1, 64), (2, 1, 64), (3, 1, 96)])
@pytest.mark.parametrize("M", [1, 70])
@pytest.mark.parametrize("act", FAR)
def test_far_below_zero(wz, forced, act, M, plan):
    forced(*plan)
    N, K = 1032, 8
    x, w = torch.zeros((M, K), dtype=torch.bfloat16, device="cuda"), torch.ones((N, K), dtype=torch.bfloat16, device="cuda")
    p = torch.linspace(*FAR[act], N, device="cuda")
    one = torch.ones(N, device="cuda")
    y = ref.act(p.double(), act)
    off = ref.FORM * y.abs() + ref.TINY
    assert float(y.abs().max()) > 2.0 ** -120
    want = tuple(t.expand(M, N) for t in (y, ref.rounded(y, off)))
    ref.check(wz.wz_linear(x, w, p, act=act), want, "y")
    ref.check(wz.wz_gated(x, w, w, p, one, act=act), want, "h")
    # the up projection's gradient, from products formed again and from kept ones (in bf16)
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    dy[M // 2] = 1.0
    kw = dict(act=act, need_x=False, need_w=False, need_b=True)
    ref.check(wz.wz_gated_backward(dy, x, w, w, b_gate=p, b_up=one, **kw)[4], (y, off), "db_up")
    gate = p.bfloat16().expand(M, N).contiguous()
    y = ref.act(gate[0].double(), act)
    got = wz.wz_gated_backward(dy, x, w, w, gate=gate, up=torch.ones_like(gate), **kw)[4]
    ref.check(got, (y, ref.FORM * y.abs() + ref.TINY), "db_up, kept")
