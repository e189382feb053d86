"""A layer's matrix products and their gradients on the GPU against 64 bits, element by element.

The bounds are derived in layer_reference.py.  Rows are slices of wider buffers whose other elements are NaN: what is
read from there spoils a result, and what is written there is seen.
"""

import pytest
import torch

import layer_reference as ref

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
    """Calls of the bounds-checked build with a kernel of the test's choice."""
    with wz.checked_library():
        yield wz._lib.wz_check_mm_plan
        wz._lib.wz_check_mm_plan(0, 1, 64)


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


class Layer:
    """Inputs of one or two weights."""

    def __init__(self, M, N, K, both, bias, pad, seed):
        g = gen(seed)
        self.M, self.N, self.K, self.pad, self.g = M, N, K, pad, g
        self.x = ref.random_rows(M, K, 1.0, g, pad)
        self.w = [ref.random_rows(N, K, 1.5 / K ** 0.5, g, pad) for _ in range(both)]
        self.b = [0.3 * torch.randn(N, generator=g, device="cuda") if bias else None for _ in range(both)]
        self.dy = ref.random_rows(M, N, 0.1, g, pad)
        self.pre = [ref.random_rows(M, N, 1.5, g, pad) for _ in range(both)]
        self.status = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.made = []

    def out(self, n, width):
        m, buffer = ref.rows(n, width, self.pad, "cuda")
        self.made.append((m, buffer))
        return m

    def done(self):
        torch.cuda.synchronize()
        assert int(self.status.item()) == 0
        for m, buffer in self.made:
            assert ref.untouched(m, buffer), "written outside of the rows"


# sizes where tiles, boxes, vectors and rows end: M, N, K
SIZES = [
    (1, 1, 1), (1, 64, 64), (1, 300, 520), (2, 7, 9), (3, 8, 1000), (5, 1000, 8), (16, 128, 64), (17, 129, 65),
    (31, 96, 33), (32, 257, 127), (33, 31, 449), (64, 512, 1152), (65, 255, 256), (100, 640, 4100), (127, 127, 127),
    (129, 385, 191), (200, 256, 2048), (255, 72, 577), (257, 1, 300), (300, 520, 31), (333, 896, 640), (513, 130, 1),
    (577, 1152, 1160), (1000, 77, 3), (1025, 513, 511),
]


def linear(wz, M, N, K, act):
    s = Layer(M, N, K, 1, bias=(M + N) % 2 == 0, pad=(N % 3) * 8, seed=M + N + K)
    residual = ref.random_rows(M, N, 2.0, s.g, 8) if (M + K) % 2 else None
    out, pre = s.out(M, N), s.out(M, N)
    got = wz.wz_linear(s.x, s.w[0], s.b[0], act=act, residual=residual, out=out, pre=pre, device_status=s.status)
    s.done()
    want, kept = ref.linear(s.x, s.w[0], s.b[0], act, residual)
    ref.check(got, want, "y")
    ref.check(pre, kept, "pre")
    # without the kept product, and with an output of the call's own: the same bits
    again = wz.wz_linear(s.x, s.w[0], s.b[0], act=act, residual=residual)
    assert torch.equal(again, got)


def gated(wz, M, N, K, act):
    s = Layer(M, N, K, 2, bias=(M + N) % 2 == 0, pad=(N % 3) * 8, seed=M + N + K)
    out, gate, up = s.out(M, N), s.out(M, N), s.out(M, N)
    got = wz.wz_gated(s.x, *s.w, *s.b, act=act, out=out, gate=gate, up=up, device_status=s.status)
    s.done()
    want, g, u = ref.gated(s.x, *s.w, *s.b, act)
    ref.check(got, want, "h")
    ref.check(gate, g, "gate")
    ref.check(up, u, "up")
    assert torch.equal(wz.wz_gated(s.x, *s.w, *s.b, act=act), got)


def linear_backward(wz, M, N, K, act, kept):
    s = Layer(M, N, K, 1, bias=(M + N) % 2 == 0, pad=(N % 3) * 8, seed=M + N + K)
    pre = s.pre[0] if kept else None
    dx, dw, db = s.out(M, K), s.out(N, K), torch.full((N,), float("nan"), device="cuda")
    wz.wz_linear_backward(s.dy, s.x, s.w[0], act=act, pre=pre, bias=s.b[0], need_b=True, dx=dx, dw=dw, db=db,
                          device_status=s.status)
    s.done()
    delta = ref.linear_delta(s.dy, s.x, s.w[0], s.b[0], pre, act)
    want_x, [want_w], [want_b] = ref.gradients(s.x, [delta], s.w, exact_delta=act == "none")
    ref.check(db, want_b, "db")
    ref.check(dx, want_x, "dx")
    ref.check(dw, want_w, "dw")


def gated_backward(wz, M, N, K, act, kept):
    s = Layer(M, N, K, 2, bias=(M + N) % 2 == 0, pad=(N % 3) * 8, seed=M + N + K)
    gate, up = s.pre if kept else (None, None)
    dx, dws = s.out(M, K), [s.out(N, K), s.out(N, K)]
    dbs = [torch.full((N,), float("nan"), device="cuda") for _ in range(2)]
    wz.wz_gated_backward(s.dy, s.x, *s.w, act=act, gate=gate, up=up, b_gate=s.b[0], b_up=s.b[1], need_b=True, dx=dx,
                         dw_gate=dws[0], dw_up=dws[1], db_gate=dbs[0], db_up=dbs[1], device_status=s.status)
    s.done()
    deltas = ref.gated_delta(s.dy, s.x, *s.w, *s.b, gate, up, act)
    want_x, want_w, want_b = ref.gradients(s.x, deltas, s.w)
    for i, name in enumerate(("gate", "up")):
        ref.check(dbs[i], want_b[i], "db_" + name)
        ref.check(dws[i], want_w[i], "dw_" + name)
    ref.check(dx, want_x, "dx")


@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_forward(wz, M, N, K, act):
    linear(wz, M, N, K, act)
    gated(wz, M, N, K, act)


@pytest.mark.parametrize("kept", [True, False])
@pytest.mark.parametrize("act", ref.ACTS)
@pytest.mark.parametrize("M,N,K", SIZES)
def test_backward(wz, M, N, K, act, kept):
    linear_backward(wz, M, N, K, act, kept)
    gated_backward(wz, M, N, K, act, kept)


@pytest.mark.parametrize("M,N,K", [(5, 200, 4200), (150, 130, 4099), (300, 520, 5000), (700, 300, 14336)])
def test_long_sums_formed_again(wz, M, N, K):
    """Products of more than 4,096 terms for their slopes: a bias gradient, a sum of M slopes of them in fp32, within 1e-5 of
    64 bits in norm (what 16 products cut off, 2^-24 of the sum at most, K / 16 times over half of K, stays below)."""
    act = "silu"
    s = Layer(M, N, K, 2, bias=True, pad=0, seed=K)
    linear_backward(wz, M, N, K, act, False)
    gated_backward(wz, M, N, K, act, False)
    got = wz.wz_gated_backward(s.dy, s.x, *s.w, act=act, b_gate=s.b[0], b_up=s.b[1], need_b=True, need_x=False, need_w=False)
    for (d, _), db in zip(ref.gated_delta(s.dy, s.x, *s.w, *s.b, None, None, act), got[3:]):
        assert float((db.double() - d.sum(0)).norm() / d.sum(0).norm()) < 1e-5


# persistent pairs of SMs; tiles on one SM and on pairs: one share of K, several, narrow and wide row tiles
PLANS = [(1, 1, 64), (2, 1, 64), (2, 2, 16), (2, 3, 208), (2, 8, 48), (2, 5, 176), (2, 1, 256),
         (3, 1, 96), (3, 2, 32), (3, 4, 192), (3, 3, 256)]


@pytest.mark.parametrize("plan", PLANS)
@pytest.mark.parametrize("M,N,K", SIZES[::2])
def test_every_kernel(wz, forced, M, N, K, plan):
    forced(*plan)
    act = ref.ACTS[(M + N + K) % 4]
    linear(wz, M, N, K, act)
    gated(wz, M, N, K, act)
    for kept in (True, False):
        linear_backward(wz, M, N, K, act, kept)
        gated_backward(wz, M, N, K, act, kept)


@pytest.mark.parametrize("plan", [(0, 1, 64), (1, 1, 64), (2, 2, 64), (3, 1, 96)])
@pytest.mark.parametrize("M", [1, 33, 70])
def test_bias_gradients_of_infinite_products(wz, forced, M, plan):
    """A weight that is infinite: the products are, and GELU's slope there is 1.  A tile's rows behind the last one, whose
    products with it are not numbers, have no part in the sums."""
    forced(*plan)
    g = gen(M)
    N, K, bad = 130, 64, 5
    x, (w, wu), dy = ref.random_rows(M, K, 1.0, g), (ref.random_rows(N, K, 0.2, g) for _ in range(2)), ref.random_rows(M, N, 0.1, g)
    x[:, 3] = 1.0
    dy[:, bad] = dy[:, bad].abs()
    w[bad, 3] = float("inf")
    large = w.clone()
    large[bad, 3] = 2.0 ** 60   # the same slopes
    db = wz.wz_linear_backward(dy, x, w, act="gelu", need_x=False, need_w=False, need_b=True)[2]
    d, e = ref.linear_delta(dy, x, large, None, None, "gelu")
    e[:, bad] = ref.FORM * dy[:, bad].double().abs()
    ref.check(db, ref.gradients(x, [(d, e)], [large])[2][0], "db")
    got = wz.wz_gated_backward(dy, x, w, wu, act="gelu", need_x=False, need_w=False, need_b=True)[3:]
    (dg, eg), (du, eu) = ref.gated_delta(dy, x, large, wu, None, None, None, None, "gelu")
    u, err = ref.product(x, wu)
    eg[:, bad] = (dy.double().abs() * (err + 2 * ref.FORM * u.abs()))[:, bad]
    ref.check(got[0], ref.gradients(x, [(dg, eg)], [large])[2][0], "db_gate")
    keep = torch.arange(N, device="cuda") != bad
    want, bound = ref.gradients(x, [(du, eu)], [large])[2][0]
    ref.check(got[1][keep], (want[keep], bound[keep]), "db_up")
    assert float(got[1][bad]) == float("inf")


@pytest.mark.parametrize("M,N,K", [(3001, 700, 320), (500, 20000, 40), (1100, 20000, 40), (2500, 130, 1000), (1024, 97, 8), (1500, 96, 9)])
def test_where_bias_gradients_are_added_up(wz, M, N, K):
    """Beside the products, by a kernel of their own, and from sums over some rows: more rows and columns of dy than fit
    into one of them."""
    linear_backward(wz, M, N, K, "none", False)
    linear_backward(wz, M, N, K, "silu", True)
    s = Layer(M, N, K, 1, bias=False, pad=8, seed=M)
    for kw in (dict(need_x=False), dict(need_w=False), dict(need_x=False, need_w=False)):
        db = wz.wz_linear_backward(s.dy, s.x, s.w[0], need_b=True, **kw)[2]
        ref.check(db, ref.gradients(s.x, [(s.dy.double(), torch.zeros_like(s.dy).double())], s.w, True)[2][0], str(kw))
