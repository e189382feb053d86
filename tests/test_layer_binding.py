"""The layer's Python calls on the host, with stand-ins for tensors and for the library: what they refuse, what they
hand over, and on which device they call; and the reference that the GPU tests compare with."""

import contextlib
import math

import pytest
import torch

import layer_reference as ref


@pytest.fixture(scope="module")
def wz():
    import paper_2607_23265_gb300.build as build
    build.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


class Fake:
    """What the binding reads of a CUDA tensor."""

    is_cuda = True

    def __init__(self, *shape, dtype=torch.bfloat16, device=1, stride=None, contiguous=True, at=1 << 20):
        self.shape, self.dtype, self._device, self._contiguous = torch.Size(shape), dtype, device, contiguous
        self._stride, self._at = stride, at
        self.nbytes = dtype.itemsize * torch.Size(shape).numel()
        self.device = torch.device("cuda", device if device >= 0 else 0)

    def stride(self):
        if self._stride:
            return self._stride
        s = [1]
        for n in self.shape[:0:-1]:
            s.insert(0, s[0] * n)
        return tuple(s)

    def dim(self):
        return len(self.shape)

    def get_device(self):
        return self._device

    def is_contiguous(self):
        return self._contiguous

    def data_ptr(self):
        return self._at


class Stream:
    cuda_stream = 0


F = lambda *shape, **kw: Fake(*shape, **kw)  # noqa: E731
V = lambda n, **kw: Fake(n, dtype=torch.float32, **kw)  # noqa: E731
M, N, K = 6, 24, 16
ARGS = {
    "wz_linear": lambda: dict(x=F(M, K), w=F(N, K), bias=V(N), residual=F(M, N), out=F(M, N), pre=F(M, N)),
    "wz_linear_backward": lambda: dict(dy=F(M, N), x=F(M, K), w=F(N, K), bias=V(N), pre=F(M, N), dx=F(M, K), dw=F(N, K),
                                       db=V(N), need_b=True),
    "wz_gated": lambda: dict(x=F(M, K), w_gate=F(N, K), w_up=F(N, K), b_gate=V(N), b_up=V(N), out=F(M, N), gate=F(M, N),
                             up=F(M, N)),
    "wz_gated_backward": lambda: dict(dout=F(M, N), x=F(M, K), w_gate=F(N, K), w_up=F(N, K), b_gate=V(N), b_up=V(N),
                                      gate=F(M, N), up=F(M, N), dx=F(M, K), dw_gate=F(N, K), dw_up=F(N, K), db_gate=V(N),
                                      db_up=V(N), need_b=True),
}


@pytest.fixture
def call(wz, monkeypatch):
    """Runs a call with the weights on device 1 and device `current` current; the devices that the library was called on
    and the arguments that it got."""
    state = {"on": 0, "seen": [], "args": None}

    class Library:
        def __getattr__(self, name):
            def fn(a):
                state["seen"].append(state["on"])
                state["args"] = a
                return 0
            return fn

    @contextlib.contextmanager
    def device(index):
        saved, state["on"] = state["on"], index
        yield
        state["on"] = saved

    monkeypatch.setattr(wz, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state["on"], raising=False)

    def run(name, current=0, **over):
        state["on"], state["seen"] = current, []
        got = getattr(wz, name)(**{**ARGS[name](), "stream": Stream, **over})
        assert state["on"] == current
        return state["seen"], state["args"], got

    return run


@pytest.mark.parametrize("name", ARGS)
@pytest.mark.parametrize("current", [0, 1])
def test_the_weights_device_is_current_in_the_call(call, name, current):
    seen, a, _ = call(name, current)
    assert seen == [1]
    assert (a.M, a.N, a.K) == (M, N, K) and a.x_stride == K


MATRICES = [(name, arg) for name, make in ARGS.items() for arg, v in make().items() if isinstance(v, Fake) and v.dim() == 2]


@pytest.mark.parametrize("name,arg", MATRICES)
@pytest.mark.parametrize("spoil", ["dtype", "device", "rows", "width", "stride", "columns"])
def test_matrices_that_do_not_fit(call, name, arg, spoil):
    good = ARGS[name]()[arg]
    n, width = good.shape
    bad = {"dtype": F(n, width, dtype=torch.float32), "device": F(n, width, device=0), "rows": F(n + 1, width),
           "width": F(n, width + 8), "stride": F(n, width, stride=(width + 4, 1)),
           "columns": F(n, width, stride=(1, n))}[spoil]
    with pytest.raises(ValueError):
        call(name, **{arg: bad})


@pytest.mark.parametrize("name,arg", [(name, arg) for name, make in ARGS.items() for arg, v in make().items()
                                      if isinstance(v, Fake) and v.dim() == 1])
def test_vectors_that_do_not_fit(call, name, arg):
    for bad in (V(N + 1), F(N), V(N, device=0), V(N, contiguous=False)):
        with pytest.raises(ValueError, match=arg):
            call(name, **{arg: bad})


def test_rows_of_a_wider_matrix_and_a_single_row(call):
    _, a, _ = call("wz_linear", x=F(M, K, stride=(40, 1)))
    assert a.x_stride == 40
    # one row: torch's stride of it says nothing
    one = dict(x=F(1, K, stride=(3, 1)), residual=F(1, N, stride=(1, 1)), out=F(1, N), pre=F(1, N))
    _, a, _ = call("wz_linear", **one)
    assert (a.M, a.x_stride, a.residual_stride) == (1, K, N)
    _, a, _ = call("wz_linear", x=F(1, 5), w=F(N, 5, stride=(8, 1)), **{k: one[k] for k in ("residual", "out", "pre")})
    assert (a.K, a.x_stride, a.w_stride) == (5, 8, 8)


def test_what_is_not_needed_is_not_asked_for(call):
    _, a, got = call("wz_linear_backward", need_x=False, need_b=False)
    assert (a.dx, a.db) == (None, None) and a.dw and got[0] is None and got[2] is None
    _, a, got = call("wz_gated_backward", need_w=False, need_b=False)
    assert (a.dw_gate, a.dw_up, a.db_gate, a.db_up) == (None,) * 4 and a.dx and got[1:] == (None,) * 4


@pytest.mark.parametrize("name", ["wz_gated", "wz_gated_backward"])
def test_gate_and_up_go_together(call, name):
    for arg in ("gate", "up"):
        with pytest.raises(ValueError, match="together"):
            call(name, **{arg: None})


@pytest.mark.parametrize("name", ["wz_linear_backward", "wz_gated_backward"])
def test_workspaces_that_the_device_cannot_use(call, name):
    for bad in (F(64, dtype=torch.uint8, device=-1), F(64, dtype=torch.uint8, device=0),
                F(64, dtype=torch.uint8, contiguous=False)):
        with pytest.raises(ValueError, match="workspace"):
            call(name, workspace=bad)
    _, a, _ = call(name, workspace=F(64, dtype=torch.uint8))
    assert a.workspace == 1 << 20 and a.workspace_bytes == 64


@pytest.mark.parametrize("name", ARGS)
def test_activations(call, name):
    for act, code in (("none", 0), ("gelu", 1), ("gelu_tanh", 2), ("silu", 3), (2, 2)):
        assert call(name, act=act)[1].act == code
    with pytest.raises(KeyError):
        call(name, act="relu")


# ---------------------------------------------------------------------------
# the reference
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("name", ref.ACTS)
def test_slopes_against_differences(name):
    x = torch.linspace(-9, 9, 3601, dtype=torch.float64)
    h = 1e-5
    steps = (ref.act(x + h, name) - ref.act(x - h, name)) / (2 * h)
    assert torch.allclose(ref.slope(x, name), steps, atol=1e-9, rtol=0)   # h^2 act''' / 6 and eps / h
    assert float(ref.slope(x, name).abs().max()) <= ref.STEEP
    second = (ref.slope(x + h, name) - ref.slope(x - h, name)) / (2 * h)
    assert float(second.abs().max()) <= ref.CURVED


def _layer(seed=0, m=9, n=7, k=11):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(s, generator=g, dtype=torch.float64)  # noqa: E731
    return r(m, k), r(n, k), r(n, k), r(n), r(n), r(m, n)


@pytest.mark.parametrize("name", ref.ACTS)
def test_gradients_against_differences(name):
    """The formulas of the backward passes, along random directions of every input."""
    x, wg, wu, bg, bu, dy = _layer()
    g = torch.Generator().manual_seed(1)
    h = 1e-6

    def plain(v):
        return (ref.act(v[0] @ v[1].T + v[2], name) * dy).sum()

    def both(v):
        return (ref.act(v[0] @ v[1].T + v[2], name) * (v[0] @ v[3].T + v[4]) * dy).sum()

    delta = ref.linear_delta(dy, x, wg, bg, None, name)
    (dx, _), [(dw, _)], [(db, _)] = ref.gradients(x, [delta], [wg], exact_delta=True)
    cases = [(plain, [x, wg, bg], [dx, dw, db])]
    deltas = ref.gated_delta(dy, x, wg, wu, bg, bu, None, None, name)
    (dx, _), dws, dbs = ref.gradients(x, deltas, [wg, wu])
    cases.append((both, [x, wg, bg, wu, bu], [dx, dws[0][0], dbs[0][0], dws[1][0], dbs[1][0]]))
    for f, values, grads in cases:
        for i, (v, d) in enumerate(zip(values, grads)):
            u = torch.randn(v.shape, generator=g, dtype=torch.float64)
            up, down = (f([w + s * h * u if i == j else w for j, w in enumerate(values)]) for s in (1, -1))
            assert math.isclose(float((up - down) / (2 * h)), float((d * u).sum()), rel_tol=1e-6, abs_tol=1e-6)


def test_the_bounds_notice_a_mistake():
    """Bounds that nothing could leave would check nothing: a slipped row, a missing bias, a wrong activation and a lost
    term are all outside them."""
    x, wg, wu, bg, bu, dy = (t.bfloat16() if t.dim() == 2 else t.float() for t in _layer(m=40, n=33, k=65))
    (y, bound), _ = ref.linear(x, wg, bg, "silu", None)
    ref.check(y.bfloat16(), (y, bound), "y")
    wrong = [y.roll(1, 0), ref.linear(x, wg, None, "silu", None)[0][0], ref.linear(x, wg, bg, "gelu", None)[0][0],
             ref.linear(x[:, :64], wg[:, :64], bg, "silu", None)[0][0]]
    deltas = ref.gated_delta(dy, x, wg, wu, bg, bu, None, None, "silu")
    dx, dw, db = ref.gradients(x, deltas, [wg, wu])
    ref.check(dx[0].bfloat16(), dx, "dx")
    pairs = [(w, (y, bound)) for w in wrong]
    pairs += [(ref.gradients(x, [deltas[1], deltas[0]], [wg, wu])[0][0], dx),
              (ref.gradients(x[:-1], [(d[:-1], e[:-1]) for d, e in deltas], [wg, wu])[1][0][0], dw[0]),
              (db[1][0] * (1 + 2.0 ** -12), db[1])]
    for got, want in pairs:
        with pytest.raises(AssertionError):
            ref.check(got, want, "wrong")
