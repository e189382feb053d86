"""The bounds-checked build looks at what a layer's products write: rows of outputs, sums over rows and shares' sums.  A
test hook has its kernels believe that there is less room than there is, all of which is allocated."""

import pytest
import torch

import layer_reference as ref

pytestmark = pytest.mark.gpu

ROWS, SUMS, SHARES = 1, 2, 4        # the last row of outputs; sums over rows, and shares' sums, but for the first
BOUNDS = 0x200
PLANS = [(1, 1, 64), (2, 1, 64), (2, 3, 48), (3, 1, 96), (3, 2, 64)]


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    assert torch.cuda.is_available()
    return m


@pytest.fixture
def checked(wz):
    with wz.checked_library():
        yield wz._lib
        wz._lib.wz_check_mm_room(0)
        wz._lib.wz_check_mm_plan(0, 1, 64)


def outputs(*shapes):
    return [ref.rows(n, width, 8, "cuda")[0] for n, width in shapes]


def operands(M, N, K, both):
    g = torch.Generator(device="cuda").manual_seed(M + N)
    x, dy = ref.random_rows(M, K, 1.0, g), ref.random_rows(M, N, 0.1, g)
    return x, dy, [ref.random_rows(N, K, K ** -0.5, g) for _ in range(both)], [ref.random_rows(M, N, 1.0, g) for _ in range(2)]


def calls(wz, M, N, K, status):
    """Every call by its name: what it writes."""
    x, dy, (w, u), (gate, up) = operands(M, N, K, 2)
    db = lambda: torch.full((N,), float("nan"), device="cuda")  # noqa: E731

    def linear():
        out, pre = outputs((M, N), (M, N))
        wz.wz_linear(x, w, act="gelu", out=out, pre=pre, device_status=status)
        return [out, pre]

    def gated():
        out, g, p = outputs((M, N), (M, N), (M, N))
        wz.wz_gated(x, w, u, out=out, gate=g, up=p, device_status=status)
        return [out, g, p]

    def linear_backward(pre, **kw):
        dx, dw = outputs((M, K), (N, K))
        wz.wz_linear_backward(dy, x, w, act="gelu", pre=pre, need_b=True, dx=dx, dw=dw, db=db(), device_status=status, **kw)
        return [t for t, need in ((dx, True), (dw, kw.get("need_w", True))) if need]

    def gated_backward(kept):
        dx, dw, dw2 = outputs((M, K), (N, K), (N, K))
        wz.wz_gated_backward(dy, x, w, u, gate=gate if kept else None, up=up if kept else None, need_b=True, dx=dx, dw_gate=dw,
                             dw_up=dw2, db_gate=db(), db_up=db(), device_status=status)
        return [dx, dw, dw2]

    return {"linear": linear, "gated": gated, "linear_backward kept": lambda: linear_backward(gate),
            "linear_backward again": lambda: linear_backward(None), "dx alone": lambda: linear_backward(gate, need_w=False),
            "gated_backward kept": lambda: gated_backward(True), "gated_backward again": lambda: gated_backward(False)}


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("M,N,K", [(1, 40, 200), (70, 300, 520), (300, 130, 260)])
def test_rows_behind_the_last_are_not_written(wz, checked, M, N, K, plan):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    checked.wz_check_mm_plan(*plan)
    for name, call in calls(wz, M, N, K, status).items():
        status.zero_()
        checked.wz_check_mm_room(0)
        assert not any(bool(torch.isnan(t.float()).any()) for t in call()) and int(status) == 0, name
        checked.wz_check_mm_room(ROWS)
        made = call()
        assert int(status) == BOUNDS, name
        for t in made:
            assert bool(torch.isnan(t[-1].float()).all()), name


@pytest.mark.parametrize("plan", PLANS)
def test_sums_behind_the_last_are_not_written(wz, checked, plan):
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    checked.wz_check_mm_plan(*plan)
    for name, call in calls(wz, 300, 130, 260, status).items():
        if "backward" in name:
            status.zero_()
            checked.wz_check_mm_room(SUMS)
            call()
            assert int(status) == BOUNDS, name


def test_shares_behind_the_last_are_not_written(wz, checked):
    """150,000 rows: three shares of the weights' gradients at least."""
    M, N, K = 150000, 72, 40
    x, dy, (w, u), (gate, up) = operands(M, N, K, 2)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for what in (0, SHARES):
        checked.wz_check_mm_room(what)
        for call in (lambda **kw: wz.wz_linear_backward(dy, x, w, need_x=False, **kw),
                     lambda **kw: wz.wz_gated_backward(dy, x, w, u, gate=gate, up=up, need_x=False, **kw)):
            status.zero_()
            call(device_status=status)
            assert int(status) == (BOUNDS if what else 0)
            call()                                    # without a status word too
    torch.cuda.synchronize()
