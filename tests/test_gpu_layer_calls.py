"""How a layer's products are called: streams, graphs, threads, places, empty and odd calls, runs of them together."""

import contextlib
import ctypes as C
import threading

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


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def rows(n, width, gain, g, pad=0):
    return ref.random_rows(n, width, gain, g, pad)


class Block:
    """A gated feed-forward block of M rows: x [M, K] -> h [M, N] -> y [M, K] = x + h Wd^T."""

    def __init__(self, M, K, N, seed, act="silu"):
        g = gen(seed)
        self.M, self.K, self.N, self.act = M, K, N, act
        self.x, self.dy = rows(M, K, 1.0, g), rows(M, K, 0.1, g)
        self.wg, self.wu = rows(N, K, 1.5 / K ** 0.5, g), rows(N, K, 1.5 / K ** 0.5, g)
        self.wd = rows(K, N, 1.5 / N ** 0.5, g)
        self.bg, self.bu, self.bd = (0.3 * torch.randn(n, generator=g, device="cuda") for n in (N, N, K))

    def forward(self, wz, **kw):
        gate, up = (torch.empty((self.M, -(-self.N // 8) * 8), dtype=torch.bfloat16, device="cuda")[:, :self.N]
                    for _ in range(2))
        h = wz.wz_gated(self.x, self.wg, self.wu, self.bg, self.bu, act=self.act, gate=gate, up=up, **kw)
        y = wz.wz_linear(h, self.wd, self.bd, residual=self.x, **kw)
        return gate, up, h, y

    def backward(self, wz, gate, up, h, **kw):
        dh, dwd, dbd = wz.wz_linear_backward(self.dy, h, self.wd, need_b=True, **kw)
        dx, dwg, dwu, dbg, dbu = wz.wz_gated_backward(dh, self.x, self.wg, self.wu, act=self.act, gate=gate, up=up,
                                                      b_gate=self.bg, b_up=self.bu, need_b=True, **kw)
        return dh, dwd, dbd, dx, dwg, dwu, dbg, dbu


@pytest.mark.parametrize("M,K,N,act", [(1, 64, 256, "silu"), (37, 200, 333, "gelu"), (300, 512, 1000, "gelu_tanh"),
                                       (1000, 384, 640, "silu")])
def test_a_block_forward_and_backward(wz, M, K, N, act):
    """Each call against 64 bits, from what the calls before it have left."""
    b = Block(M, K, N, seed=M, act=act)
    gate, up, h, y = b.forward(wz)
    want, g, u = ref.gated(b.x, b.wg, b.wu, b.bg, b.bu, act)
    for got, w, name in ((h, want, "h"), (gate, g, "gate"), (up, u, "up"),
                         (y, ref.linear(h, b.wd, b.bd, "none", b.x)[0], "y")):
        ref.check(got, w, name)
    dh, dwd, dbd, dx, dwg, dwu, dbg, dbu = b.backward(wz, gate, up, h)
    want_x, [want_w], [want_b] = ref.gradients(h, [ref.linear_delta(b.dy, h, b.wd, None, None, "none")], [b.wd], True)
    ref.check(dh, want_x, "dh")
    ref.check(dwd, want_w, "dwd")
    ref.check(dbd, want_b, "dbd")
    deltas = ref.gated_delta(dh, b.x, b.wg, b.wu, b.bg, b.bu, gate, up, act)
    want_x, want_w, want_b = ref.gradients(b.x, deltas, [b.wg, b.wu])
    for got, w, name in ((dx, want_x, "dx"), (dwg, want_w[0], "dwg"), (dwu, want_w[1], "dwu"), (dbg, want_b[0], "dbg"),
                         (dbu, want_b[1], "dbu")):
        ref.check(got, w, name)
    # formed again instead of kept: the same formulas from fp32 products
    again = wz.wz_gated_backward(dh, b.x, b.wg, b.wu, act=act, b_gate=b.bg, b_up=b.bu, need_b=True)
    deltas = ref.gated_delta(dh, b.x, b.wg, b.wu, b.bg, b.bu, None, None, act)
    want_x, want_w, want_b = ref.gradients(b.x, deltas, [b.wg, b.wu])
    for got, w in zip(again, (want_x, *want_w, *want_b)):
        ref.check(got, w, "formed again")


@pytest.mark.parametrize("seed", range(3))
def test_gradients_against_differences(wz, seed):
    """The gradients that the GPU gives along a random direction of each input, against differences of the loss in 64
    bits.  The loss is a sum over outputs with dy as weights; a gradient's elements are off by at most the bounds of
    layer_reference, so their product with the direction is off by at most the bounds' product with its magnitudes."""
    act = ref.ACTS[1 + seed]
    b = Block(50, 72, 96, seed, act)
    gate, up, h, y = b.forward(wz)
    dh = torch.randn((b.M, b.N), generator=gen(seed + 9), device="cuda").bfloat16()
    got = wz.wz_gated_backward(dh, b.x, b.wg, b.wu, act=act, b_gate=b.bg, b_up=b.bu, need_b=True)
    deltas = ref.gated_delta(dh, b.x, b.wg, b.wu, b.bg, b.bu, None, None, act)
    want_x, want_w, want_b = ref.gradients(b.x, deltas, [b.wg, b.wu])
    bounds = [w[1] for w in (want_x, *want_w, *want_b)]

    def loss(x, wg, wu, bg, bu):
        return (ref.act(x @ wg.T + bg, act) * (x @ wu.T + bu) * dh.double()).sum()

    values = [t.double() for t in (b.x, b.wg, b.wu, b.bg, b.bu)]
    g = gen(seed + 20)
    step = 1e-5
    for i in range(5):
        u = torch.randn(values[i].shape, generator=g, device="cuda", dtype=torch.float64)
        up_, down = (loss(*[v + s * step * u if i == j else v for j, v in enumerate(values)]) for s in (1, -1))
        slope = float((up_ - down) / (2 * step))
        along = float((got[i].double() * u).sum())
        bound = float((bounds[i] * u.abs()).sum()) + 1e-6 * (1 + abs(slope))
        assert abs(along - slope) <= bound, (i, along, slope, bound)


def test_the_residual_may_be_the_output(wz):
    g = gen(3)
    for M, K, N in ((1, 512, 256), (40, 300, 130), (700, 256, 520)):
        x, w, r = rows(M, K, 1.0, g), rows(N, K, 1.5 / K ** 0.5, g), rows(M, N, 2.0, g, 8)
        want = wz.wz_linear(x, w, residual=r)
        out = wz.wz_linear(x, w, residual=r, out=r)
        assert out is r and torch.equal(r, want)


def test_no_rows(wz):
    empty = torch.empty((0, 64), dtype=torch.bfloat16, device="cuda")
    w = rows(128, 64, 1.0, gen(1))
    assert wz.wz_linear(empty, w).shape == (0, 128) and wz.wz_gated(empty, w, w).shape == (0, 128)
    dy = empty.new_empty((0, 128))
    dx, dw, db = wz.wz_linear_backward(dy, empty, w, act="gelu", need_b=True)
    assert dx.shape == (0, 64) and not dw.any() and not db.any() and dw.shape == (128, 64) and db.shape == (128,)
    got = wz.wz_gated_backward(dy, empty, w, w, need_b=True)
    assert got[0].shape == (0, 64) and not any(bool(t.any()) for t in got[1:])
    dw, buffer = ref.rows(5, 13, 8, "cuda")
    wz.wz_linear_backward(empty.new_empty((0, 8))[:, :5], empty[:, :13], rows(5, 13, 1.0, gen(2), 8), need_x=False, dw=dw)
    assert not dw.any() and ref.untouched(dw, buffer)


@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_what_is_not_finite_stays_in_its_row(wz, bad):
    g = gen(4)
    for M, N, K in ((20, 200, 512), (600, 300, 320)):
        x, w = rows(M, K, 1.0, g), rows(N, K, 1.5 / K ** 0.5, g)
        clean = wz.wz_linear(x, w, act="gelu")
        x2 = x.clone()
        x2[7, 5] = bad
        got = wz.wz_linear(x2, w, act="gelu")
        keep = torch.arange(M, device="cuda") != 7
        assert torch.equal(got[keep], clean[keep])
        # each output of the row has the bad number as a term; GELU takes -infinity to 0 or NaN
        assert not torch.isfinite(got[7][w[:, 5] > 0]).any()
        # backward: dW has it in column 5 alone, dx nowhere
        dy = rows(M, N, 0.1, g)
        dx, dw, _ = wz.wz_linear_backward(dy, x2, w)
        dx0, dw0, _ = wz.wz_linear_backward(dy, x, w)
        other = torch.arange(K, device="cuda") != 5
        assert torch.equal(dx, dx0) and torch.equal(dw[:, other], dw0[:, other]) and not torch.isfinite(dw[:, 5]).any()


def test_activations_of_large_numbers(wz):
    """Products of up to 2^100: values and slopes are what the formulas' limits are, never NaN."""
    x = torch.tensor([[1.0], [-1.0]], device="cuda").bfloat16().expand(2, 8).contiguous()
    w = torch.zeros((64, 8), dtype=torch.bfloat16, device="cuda")
    w[:, 0] = torch.tensor([2.0 ** e for e in range(-20, 44)]).cuda()
    w[60:, 0] = torch.tensor([2.0 ** 60, 2.0 ** 70, 2.0 ** 90, 2.0 ** 100]).cuda()
    for act in ref.ACTS:
        (y, bound), _ = ref.linear(x, w, None, act, None)
        ref.check(wz.wz_linear(x, w, act=act), (y, bound), act)
        dy = torch.ones((2, 64), dtype=torch.bfloat16, device="cuda")
        _, _, db = wz.wz_linear_backward(dy[:1], x[:1], w, act=act, need_x=False, need_w=False, need_b=True)
        p = w[:, 0].double()
        assert torch.allclose(db.double(), ref.slope(p.clamp(max=1e6), act), atol=2e-5)
        _, _, db = wz.wz_linear_backward(dy[:1], x[1:], w, act=act, need_x=False, need_w=False, need_b=True)
        assert torch.allclose(db.double(), ref.slope(-p.clamp(max=1e6), act), atol=2e-5)


def test_rows_past_31_bits(wz):
    """Offsets of x, residual, dy, dx and the outputs that need more than 32 bits."""
    M, N, K = 2100, 72, 64
    wide = 1 << 20                                            # elements from row to row: 4.4 GB in all
    g = gen(6)
    big = torch.empty((M, wide), dtype=torch.bfloat16, device="cuda")
    col = iter(range(0, wide, 4096))

    def place(t):
        c = next(col)
        v = big[:, c:c + t.shape[1]]
        v.copy_(t)
        return v

    x, dy, r = rows(M, K, 1.0, g), rows(M, N, 0.1, g), rows(M, N, 1.0, g)
    w, w2 = rows(N, K, 0.2, g), rows(N, K, 0.2, g)
    X, DY, R, OUT, PRE, UP, DX = (place(t) for t in (x, dy, r, dy, dy, dy, x))
    assert torch.equal(wz.wz_linear(X, w, act="gelu", residual=R, out=OUT, pre=PRE), wz.wz_linear(x, w, act="gelu", residual=r))
    wz.wz_linear_backward(DY, X, w, act="gelu", pre=PRE, dx=DX)
    assert torch.equal(DX, wz.wz_linear_backward(dy, x, w, act="gelu", pre=PRE.contiguous())[0])
    wz.wz_linear_backward(DY, X, w, act="gelu", dx=DX)
    assert torch.equal(DX, wz.wz_linear_backward(dy, x, w, act="gelu")[0])
    assert torch.equal(wz.wz_gated(X, w, w2, out=OUT, gate=PRE, up=UP), wz.wz_gated(x, w, w2))
    wz.wz_gated_backward(DY, X, w, w2, gate=PRE, up=UP, dx=DX)
    assert torch.equal(DX, wz.wz_gated_backward(dy, x, w, w2, gate=PRE.contiguous(), up=UP.contiguous())[0])


@pytest.mark.parametrize("M,N,K", [(70000, 8, 8), (5, 65536, 16), (16, 8, 65536), (140000, 3, 65)])
def test_long_and_wide(wz, M, N, K):
    g = gen(M)
    x, w, dy = rows(M, K, 1.0, g), rows(N, K, 1.0 / K ** 0.5, g), rows(M, N, 0.1, g)
    b = torch.randn(N, generator=g, device="cuda")
    want, _ = ref.linear(x, w, b, "silu", None)
    ref.check(wz.wz_linear(x, w, b, act="silu"), want, "y")
    dx, dw, db = wz.wz_linear_backward(dy, x, w, act="silu", bias=b, need_b=True)
    delta = ref.linear_delta(dy, x, w, b, None, "silu")
    want_x, [want_w], [want_b] = ref.gradients(x, [delta], [w])
    ref.check(dx, want_x, "dx")
    ref.check(dw, want_w, "dw")
    ref.check(db, want_b, "db")


def all_calls(wz, b, ws=None, **kw):
    """Every entry point once, and what they return."""
    ws = {} if ws is None else ws
    gate, up, h, y = b.forward(wz, **kw)
    dh, dwd, dbd = wz.wz_linear_backward(b.dy, h, b.wd, act="gelu", pre=y, need_b=True, workspace=ws.get("linear"), **kw)
    got = wz.wz_gated_backward(dh, b.x, b.wg, b.wu, act=b.act, gate=gate, up=up, need_b=True, workspace=ws.get("gated"), **kw)
    again = wz.wz_gated_backward(dh, b.x, b.wg, b.wu, act=b.act, b_gate=b.bg, b_up=b.bu, need_b=True,
                                 workspace=ws.get("gated"), **kw)
    return [gate, up, h, y, dh, dwd, dbd, *got, *again]


def workspaces(wz, b):
    return {"linear": torch.empty(wz.wz_linear_backward_workspace_size(b.M, b.N, b.K), dtype=torch.uint8, device="cuda"),
            "gated": torch.empty(wz.wz_gated_backward_workspace_size(b.M, b.K, b.N), dtype=torch.uint8, device="cuda")}


SHAPES = [(1, 512, 1024), (50, 1152, 700), (577, 320, 520), (1500, 264, 300)]


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_equal_calls_give_equal_bits(wz, M, K, N):
    """With the library's workspace, with a caller's that holds anything, and again."""
    b = Block(M, K, N, seed=M)
    first = all_calls(wz, b)
    ws = workspaces(wz, b)
    for fill in (0xFF, 0x7F, 0):
        for t in ws.values():
            t.fill_(fill)
        for one, two in zip(first, all_calls(wz, b, ws)):
            assert torch.equal(one, two)


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_the_checked_build_agrees(wz, M, K, N):
    b = Block(M, K, N, seed=M)
    first = all_calls(wz, b)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with wz.checked_library():
        for one, two in zip(first, all_calls(wz, b, device_status=status)):
            assert torch.equal(one, two)
    assert int(status) == 0


@pytest.mark.parametrize("M,K,N", [(1, 512, 1024), (40, 320, 700), (700, 256, 384)])
def test_weights_that_the_call_before_has_just_written(wz, M, K, N):
    """The first weights are sent for early; what a product takes is what the grid in front of it has left there."""
    g = gen(N)
    x, left = rows(M, K, 1.0, g), [rows(N, 64, 0.4, g) for _ in range(6)]
    right = rows(K, 64, 0.3, g)
    w, first = torch.zeros((N, K), dtype=torch.bfloat16, device="cuda"), rows(M, N, 1.0, g)
    dy, out = first, []
    for a in left:
        wz.wz_linear(a, right, out=w)
        y, h = wz.wz_linear(x, w), wz.wz_gated(x, w, w)
        wz.wz_linear(a, right, out=w)
        out.append((y, h, wz.wz_linear_backward(dy, x, w, need_w=False)[0]))
        dy = y
    torch.cuda.synchronize()
    dy = first
    for a, (y, h, dx) in zip(left, out):
        w = wz.wz_linear(a, right)
        torch.cuda.synchronize()
        assert torch.equal(y, wz.wz_linear(x, w)) and torch.equal(h, wz.wz_gated(x, w, w))
        assert torch.equal(dx, wz.wz_linear_backward(dy, x, w, need_w=False)[0])
        dy = y


@pytest.mark.parametrize("M,K,N", SHAPES)
def test_captured_and_replayed(wz, M, K, N):
    """Two graphs that share a workspace, each replayed on new contents, in turn."""
    blocks = [Block(M, K, N, seed=s) for s in (1, 2)]
    ws = workspaces(wz, blocks[0])
    s = torch.cuda.Stream()
    graphs, outs = [], []
    with torch.cuda.stream(s):
        all_calls(wz, blocks[0], ws)
        torch.cuda.synchronize()
        for b in blocks:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g, stream=s):
                outs.append(all_calls(wz, b, ws))
            graphs.append(g)
    for seed in (5, 6):
        for i, b in enumerate(blocks):
            fresh = Block(M, K, N, seed=10 * seed + i)
            b.x.copy_(fresh.x)
            b.wg.copy_(fresh.wg)
            b.dy.copy_(fresh.dy)
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for g in graphs:
                g.replay()
        torch.cuda.synchronize()
        for b, out in zip(blocks, outs):
            for one, two in zip(out, all_calls(wz, b)):
                assert torch.equal(one, two)


def test_two_streams_and_two_threads(wz):
    """Calls that overlap, on streams and threads of their own."""
    blocks = [Block(M, 768, 1500, seed=M) for M in (64, 700)]
    want = [all_calls(wz, b) for b in blocks]
    torch.cuda.synchronize()
    got, errors = [None, None], []

    def work(i):
        try:
            s = torch.cuda.Stream()
            with torch.cuda.stream(s):
                for _ in range(10):
                    got[i] = all_calls(wz, blocks[i], workspaces(wz, blocks[i]))
            s.synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors
    for one, two in zip(want, got):
        for a, b in zip(one, two):
            assert torch.equal(a, b)


def test_a_given_stream_waits_for_its_own_work(wz):
    """On a stream other than the current one: inputs made there, late, are seen."""
    b = Block(300, 512, 640, seed=8)
    want = all_calls(wz, b)
    side = torch.cuda.Stream()
    x = b.x.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        b.x.zero_()
        big = torch.randn((4096, 4096), device="cuda")
        for _ in range(20):
            big = big @ big * 1e-3
        b.x.copy_(x)
    got = all_calls(wz, b, stream=side)
    side.synchronize()
    for one, two in zip(want, got):
        assert torch.equal(one, two)


def test_outputs_do_not_come_from_another_streams_memory(wz):
    b = Block(64, 256, 512, seed=9)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    torch.cuda.synchronize()
    freed = torch.empty((b.M, b.N), dtype=torch.bfloat16, device="cuda")
    address = freed.data_ptr()
    del freed
    got = wz.wz_gated(b.x, b.wg, b.wu, stream=side)
    assert got.data_ptr() != address
    side.synchronize()


@contextlib.contextmanager
def impatient(wz, plan):
    """The checked library with a plan of the test's choice, whose waits give up after a nanosecond."""
    lib = C.CDLL(wz.LIB_CHECKED_PATH)
    lib.wz_check_mm_wait.argtypes, lib.wz_check_mm_wait.restype = [C.c_uint64], None
    with wz.checked_library():
        wz._lib.wz_check_mm_plan(*plan)
        lib.wz_check_mm_wait(1)
        try:
            yield
        finally:
            torch.cuda.synchronize()
            lib.wz_check_mm_wait(0)
            wz._lib.wz_check_mm_plan(0, 1, 64)


@pytest.mark.parametrize("plan", [(1, 1, 64), (2, 1, 64), (2, 4, 48), (3, 1, 96), (3, 2, 192)])
def test_calls_that_give_up_end_and_the_next_is_right(wz, plan):
    b = Block(300, 2048, 1100, seed=11)
    want = all_calls(wz, b)
    torch.cuda.synchronize()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    with impatient(wz, plan):
        all_calls(wz, b, device_status=status)
        torch.cuda.synchronize()
        assert int(status) & wz.STATUS_WAIT_TIMEOUT
    status.zero_()
    for one, two in zip(want, all_calls(wz, b, device_status=status)):
        assert torch.equal(one, two)
    assert int(status) == 0
