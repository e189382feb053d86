"""Gradients of the input alone, as layers with frozen weights need them: dx may take the kernel for few tiles, with weights
whose rows are K and, behind a gated product, two products in one sum."""

import pytest
import torch

import layer_reference as ref
from test_gpu_layer import PLANS, SIZES, Layer, gated, gated_backward, linear, linear_backward

pytestmark = pytest.mark.gpu


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


# N in pieces of 64: 2, 3, 5, 7 and 9 of them twice, so that shares of K go over from one product to the other
ODD = [(40, 97, 200), (70, 190, 300), (130, 300, 64), (33, 420, 520), (200, 577, 130)]


def frozen(wz, M, N, K, act):
    s = Layer(M, N, K, 2, bias=(M + N) % 2 == 0, pad=(N % 3) * 8, seed=M + N + K)
    for kept in (True, False):
        pre = s.pre[0] if kept else None
        dx, db = s.out(M, K), torch.full((N,), float("nan"), device="cuda")
        got = wz.wz_linear_backward(s.dy, s.x, s.w[0], act=act, pre=pre, bias=s.b[0], need_w=False, need_b=True, dx=dx, db=db,
                                    device_status=s.status)
        assert got[0] is dx and got[1] is None
        s.done()
        want_x, _, [want_b] = ref.gradients(s.x, [ref.linear_delta(s.dy, s.x, s.w[0], s.b[0], pre, act)], s.w[:1],
                                            exact_delta=act == "none")
        ref.check(dx, want_x, "dx")
        ref.check(db, want_b, "db")
        gate, up = s.pre if kept else (None, None)
        dx = s.out(M, K)
        got = wz.wz_gated_backward(s.dy, s.x, *s.w, act=act, gate=gate, up=up, b_gate=s.b[0], b_up=s.b[1], need_w=False,
                                   need_b=True, dx=dx, device_status=s.status)
        assert got[0] is dx and got[1] is None and got[2] is None
        s.done()
        want_x, _, want_b = ref.gradients(s.x, ref.gated_delta(s.dy, s.x, *s.w, *s.b, gate, up, act), s.w)
        ref.check(dx, want_x, "dx of both")
        ref.check(got[3], want_b[0], "db_gate")
        ref.check(got[4], want_b[1], "db_up")


@pytest.mark.parametrize("M,N,K", SIZES + ODD)
def test_dx_alone(wz, M, N, K):
    for act in ref.ACTS:
        frozen(wz, M, N, K, act)


@pytest.mark.parametrize("M,N,K", SIZES + ODD)
def test_dx_alone_by_every_kernel(wz, forced, M, N, K):
    for plan in PLANS:
        print(plan)
        forced(*plan)
        frozen(wz, M, N, K, ref.ACTS[(M + N + K) % 4])


@pytest.mark.parametrize("M,N,K", SIZES[1::2])
def test_every_kernel_at_the_other_sizes(wz, forced, M, N, K):
    """All calls with all gradients, at those of the odd sizes that test_gpu_layer's test of every kernel leaves out."""
    act = ref.ACTS[(M + N + K) % 4]
    for plan in PLANS:
        print(plan)
        forced(*plan)
        linear(wz, M, N, K, act)
        gated(wz, M, N, K, act)
        for kept in (True, False):
            linear_backward(wz, M, N, K, act, kept)
            gated_backward(wz, M, N, K, act, kept)
