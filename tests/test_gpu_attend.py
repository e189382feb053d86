"""wz_attend against a plain form in 64 bits.

Tolerance of an output: 2^-9 of it for its rounding to bf16 (half of the most that can be), the weights' rounding (two e4m3 numbers
of a weight, each to 2^-4 of what it stands for: 2^-8 of sum p |v|, and for weights of a tile below
2^-14 of its largest 2^-18 of that, at most 128 of them to a tile: 2^-11), and what the logits'
errors (kv_reference.attend) do to the weights, numerator and denominator."""

import math

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
    assert torch.cuda.is_available()
    return m


def compare(out, lse, host, q, table, cu, kv_len, causal, scale):
    want, wlse, mass, off = ref.attend(host, q, table, cu, kv_len, causal, scale)
    got, glse = out.cpu().double(), lse.cpu().double()
    tol = 2.0 ** -9 * 1.01 * want.abs() + (2.0 ** -8 + 2.0 ** -11 + 2 * off[..., None]) * 1.05 * mass + 1e-30
    bad = (got - want).abs() > tol
    assert not bool(bad.any()), float(((got - want).abs() / tol).max())
    empty = torch.isneginf(wlse)
    assert torch.equal(torch.isneginf(glse), empty)
    assert bool((got[empty] == 0).all())
    err = (glse - wlse)[~empty].abs()
    assert bool((err <= (off + 2.0 ** -20 * wlse.abs() + 2.0 ** -19)[~empty]).all()), float(err.max())


def poison(gpu, table, kv_len, P):
    """NaN wherever no slot in use lies."""
    used = torch.zeros(gpu.k.shape[0], P, dtype=torch.bool)
    for row, n in zip(table, kv_len):
        for t in range(n):
            used[row[t // P], t % P] = True
    at = (~used).nonzero()
    for x in (gpu.k, gpu.v):
        x.view(torch.uint8)[at[:, 0].cuda(), :, at[:, 1].cuda()] = 0x7F


def run(wz, P, heads, Hq, D, new, kv_len, causal=True, seed=1, scale=None, gain=2.0, **kw):
    g = torch.Generator().manual_seed(seed)
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    table, pages = tables(kv_len, P, seed)
    host = ref.Cache(pages, heads, P, D, seed=seed)
    gpu = host.on_gpu(wz)
    poison(gpu, table, kv_len, P)
    q = (torch.randn((cu[-1], Hq, D), generator=g) * gain).to(torch.bfloat16)
    lse = torch.full((cu[-1], Hq), 7.0, device="cuda")
    out = wz.wz_attend(q.cuda(), gpu, i32(table), i32(cu), i32(kv_len), max_new=max(new), causal=causal, scale=scale,
                       lse=lse, **kw)
    compare(out, lse, host, q, table, cu, kv_len, causal, 1 / math.sqrt(D) if scale is None else scale)


FEW = [
    # page, heads, Hq, D, new, kv_len
    (16, 1, 1, 16, [1], [1]),
    (16, 2, 2, 64, [1, 1, 1], [0, 15, 17]),
    (64, 4, 28, 128, [1], [741]),
    (32, 1, 8, 128, [1, 1, 1, 1], [127, 128, 129, 257]),
    (128, 2, 32, 128, [1, 1], [1000, 3]),
    (64, 8, 32, 128, [4, 4], [700, 64]),
    (16, 3, 3, 80, [5, 1, 0, 3], [5, 40, 30, 260]),
    (32, 5, 5, 96, [8, 2], [3, 131]),            # more tokens than slots: rows that see nothing
    (64, 2, 14, 48, [2], [385]),
    (64, 2, 4, 112, [1, 0, 0, 1], [90, 0, 64, 1]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", FEW, ids=[str(i) for i in range(len(FEW))])
def test_few_rows(wz, case, causal):
    run(wz, *case, causal=causal)


MANY = [
    # page, heads, Hq, D, new, kv_len
    (64, 1, 1, 128, [17], [17]),
    (16, 2, 14, 128, [3], [3]),
    (32, 4, 28, 128, [40], [741]),
    (64, 2, 2, 64, [128, 129, 1, 0], [128, 129, 300, 50]),
    (128, 1, 3, 96, [257], [1000]),
    (16, 3, 3, 80, [300, 20], [300, 700]),
    (64, 2, 10, 48, [60, 77], [33, 0]),          # more tokens than slots: rows that see nothing
    (32, 8, 8, 112, [140], [269]),
    (128, 1, 40, 16, [1, 2], [500, 129]),        # many heads to a group
    (64, 1, 5, 128, [500], [1500]),
]


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", MANY, ids=[str(i) for i in range(len(MANY))])
def test_many_rows(wz, case, causal):
    run(wz, *case, causal=causal)


def test_rows_whose_maximum_rises(wz):
    """Logits that grow along the sequence by far more than a rescale's slack, and a negative scale."""
    for scale, seed in ((3.0, 1), (-3.0, 2)):
        run(wz, 32, 1, 2, 64, [64], [900], scale=scale, seed=seed, gain=4.0)


def test_one_long_sequence(wz):
    """Every CTA holds a piece of the same item."""
    run(wz, 128, 1, 2, 64, [1], [128 * 700 + 5])


def test_many_short_sequences(wz):
    """Many items to a CTA, some without slots or tokens."""
    kv = [(13 * b) % 300 for b in range(500)]
    run(wz, 16, 2, 4, 32, [b % 3 != 1 and 1 or 0 for b in range(500)], kv)


@pytest.mark.parametrize("spread", [0.0, 12.0])
def test_tokens_that_outweigh(wz, spread):
    """One token far above thousands of even ones, whose small weights together count as much."""
    P, D, kv = 64, 64, 4099
    table, pages = tables([kv], P, 3)
    host = ref.Cache(pages, 1, P, D, seed=6)
    host.codes["k"][:] = 0
    host.scale["k"][:] = 2.0 ** -5
    first = table[0][0]
    host.codes["k"][first, 0, 5, 0] = 256.0       # logit 8 * q0 * scale of this token, 0 of the others
    host.codes["v"][first, 0, 5] *= 2.0 ** -5
    gpu = host.on_gpu(wz)
    q = torch.zeros((1, 1, D), dtype=torch.bfloat16)
    q[0, 0, 0] = spread / 8
    lse = torch.empty((1, 1), device="cuda")
    out = wz.wz_attend(q.cuda(), gpu, i32(table), i32([0, 1]), i32([kv]), max_new=1, scale=1.0, lse=lse)
    compare(out, lse, host, q, table, [0, 1], [kv], True, 1.0)


def test_scales_far_apart(wz):
    """Neighbouring pages whose scales are 2^40 apart, for keys and for values."""
    P, D, kv = 16, 32, 300
    table, pages = tables([kv], P, 3)
    host = ref.Cache(pages, 1, P, D, seed=6)
    for j, page in enumerate(table[0]):
        host.scale["v"][page] = 2.0 ** (-45 + 40 * (j % 2))
        host.scale["k"][page] = 2.0 ** (-44 if j % 3 == 0 else -6)
    gpu = host.on_gpu(wz)
    q = torch.randn((1, 1, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    lse = torch.empty((1, 1), device="cuda")
    out = wz.wz_attend(q.cuda(), gpu, i32(table), i32([0, 1]), i32([kv]), max_new=1, lse=lse)
    compare(out, lse, host, q, table, [0, 1], [kv], True, D ** -0.5)


def nan_case(wz, heads, G, n, kv, D=64, P=32):
    """A NaN in V at a slot that only the sequence's last two tokens see."""
    table, pages = tables([kv], P, 3)
    host = ref.Cache(pages, heads, P, D, seed=6)
    q = torch.randn((n, heads * G, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    clean = host.on_gpu(wz)
    lse = torch.empty((n, heads * G), device="cuda")
    args = (i32(table), i32([0, n]), i32([kv]))
    want = wz.wz_attend(q.cuda(), clean, *args, lse=lse).clone()
    gpu = host.on_gpu(wz)
    t, c = kv - 2, 5
    gpu.v.view(torch.uint8)[table[0][t // P], :, t % P, c] = 0xFF
    got = wz.wz_attend(q.cuda(), gpu, *args)
    sees = torch.zeros(n, dtype=torch.bool)
    sees[-2:] = True
    assert bool(torch.isnan(got[sees.cuda()][..., c]).all())
    keep = torch.ones(got.shape, dtype=torch.bool)
    keep[sees, :, c] = False
    assert torch.equal(got.cpu()[keep], want.cpu()[keep])


@pytest.mark.parametrize("n", [4, 9, 150])
@pytest.mark.parametrize("kv", [40, 128, 129, 1400])
def test_nan_that_only_some_rows_see(wz, kv, n):
    nan_case(wz, 2, 2, min(n, kv), kv)


@pytest.mark.parametrize("n", [3, 30])
def test_nan_inputs(wz, n):
    """A NaN or an infinity in a query makes its row NaN, one in a key the rows that see it."""
    P, D, kv = 32, 64, 200
    table, pages = tables([kv], P, 3)
    host = ref.Cache(pages, 1, P, D, seed=6)
    q = torch.randn((n, 2, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    args = (i32(table), i32([0, n]), i32([kv]))
    want = wz.wz_attend(q.cuda(), host.on_gpu(wz), *args)
    bad = q.clone()
    bad[0, 1, 7], bad[2, 0, 3] = float("nan"), float("inf")
    got = wz.wz_attend(bad.cuda(), host.on_gpu(wz), *args)
    nan = torch.isnan(got).all(-1).cpu()
    assert nan[:3].tolist() == [[False, True], [False, False], [True, False]] and not bool(nan[3:].any())
    assert torch.equal(got.cpu()[~nan], want.cpu()[~nan])
    gpu = host.on_gpu(wz)
    t = kv - 2                                       # seen by the last two tokens
    gpu.k.view(torch.uint8)[table[0][t // P], 0, t % P, 1] = 0x7F
    got = wz.wz_attend(q.cuda(), gpu, *args)
    assert torch.isnan(got).all(-1).cpu().tolist() == [[False] * 2] * (n - 2) + [[True] * 2] * 2
    assert torch.equal(got[:n - 2], want[:n - 2])


def test_strides_workspace_and_stream(wz):
    """Queries and outputs inside wider rows, a kept workspace, another stream: the same bits."""
    P, D, kv = 64, 128, [900, 77]
    table, pages = tables(kv, P, 3)
    host = ref.Cache(pages, 2, P, D, seed=6)
    gpu = host.on_gpu(wz)
    wide = torch.randn((2, 20, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    args = (i32(table), i32([0, 1, 2]), i32(kv))
    want = wz.wz_attend(wide[:, 4:12].contiguous(), gpu, *args, max_new=1)
    ws = torch.full((wz.wz_attend_workspace_size(2, 8, D),), 255, dtype=torch.uint8, device="cuda")
    room = torch.zeros((2, 20, D), dtype=torch.bfloat16, device="cuda")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        wz.wz_attend(wide[:, 4:12], gpu, *args, max_new=1, out=room[:, 8:16], workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(room[:, 8:16], want)
    assert int(room[:, :8].abs().max()) == 0 and int(room[:, 16:].abs().max()) == 0


def test_far_pages(wz):
    """Pages past 4 GiB of codes."""
    P, heads, D = 128, 8, 128
    pages = (1 << 32) // (P * heads * D) + 3
    host = ref.Cache(3, heads, P, D, seed=6)
    small, big = host.on_gpu(wz), wz.KvCache.empty(pages, heads, P, D)
    for n in ("k", "v", "k_scale", "v_scale"):
        getattr(big, n).view(torch.uint8)[pages - 3:] = getattr(small, n).view(torch.uint8)
    q = torch.randn((1, 16, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    a = wz.wz_attend(q, small, i32([[2, 0, 1]]), i32([0, 1]), i32([300]))
    b = wz.wz_attend(q, big, i32([[pages - 1, pages - 3, pages - 2]]), i32([0, 1]), i32([300]))
    assert torch.equal(a, b)


@pytest.mark.parametrize("what", ["page", "kv", "cu"])
def test_entries_outside_are_reported(wz, what):
    """A page outside the cache is skipped, a length past the table cut, lengths of q that
    contradict T dropped; each sets the status bit."""
    P, D = 16, 32
    host = ref.Cache(6, 1, P, D, seed=6)
    gpu = host.on_gpu(wz)
    q = torch.randn((2, 1, D), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16)
    table, cu, kv = [[0, 1, 2], [3, 4, 5]], [0, 1, 2], [40, 33]
    sane = {"table": [r[:] for r in table], "kv": kv[:]}
    if what == "page":
        table[0][1] = 6
    elif what == "kv":
        kv[0], sane["kv"][0] = 49, 48
    else:
        cu = [0, 1, 3]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = torch.zeros((2, 1, D), dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((2, 1), device="cuda")
    wz.wz_attend(q.cuda(), gpu, i32(table), i32(cu), i32(kv), max_new=1, out=out, lse=lse, device_status=status)
    assert int(status) == wz.STATUS_CACHE
    if what == "page":
        # the slots of the page are not there: its sequence as two pieces, 16 and 8 slots
        short = [[0, 2], table[1]]
        compare(out, lse, host, q, [short[0] + [-1], short[1]], [0, 1, 2], [24, 33], True, D ** -0.5)
    elif what == "kv":
        compare(out, lse, host, q, sane["table"], [0, 1, 2], sane["kv"], True, D ** -0.5)
    else:
        assert int(out[1].abs().max()) == 0


def test_append_then_attend_token_by_token(wz):
    """What a decoder does: each token appended, then attending, equals the reference's own cache."""
    P, heads, Hq, D = 16, 2, 4, 64
    g = torch.Generator().manual_seed(2)
    host = ref.Cache(4, heads, P, D, seed=5)
    gpu = host.on_gpu(wz)
    table, rotation = [[2, 0, 3]], wz.rotation_table(64, D)
    for i in range(35):
        qkv = torch.randn((1, Hq + 2 * heads, D), generator=g).to(torch.bfloat16).cuda()
        q = wz.wz_kv_append(qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], gpu, i32(table), i32([0, 1]), i32([i]), max_new=1,
                            q=qkv[:, :Hq], rotation=rotation)
        lse = torch.empty((1, Hq), device="cuda")
        out = wz.wz_attend(q, gpu, i32(table), i32([0, 1]), i32([i + 1]), max_new=1, lse=lse)
        for n in "kv":
            host.codes[n] = getattr(gpu, n).cpu().double()
            host.scale[n] = getattr(gpu, n + "_scale").cpu().double()
        compare(out, lse, host, q.cpu(), table, [0, 1], [i + 1], True, D ** -0.5)


@pytest.mark.parametrize("G,n", [(1, 1), (7, 1), (4, 3)])
def test_items_in_pieces(wz, G, n):
    """Sequences from one tile to thirty, some without slots: items of one piece, of several, and
    several items to a CTA, with few and with many items."""
    for seqs, heads in ((3, 1), (30, 4)):
        kv = [0 if b % 7 == 5 else (b * 977 + 31) % 3900 + 1 for b in range(seqs)]
        run(wz, 128, heads, heads * G, 64, [n] * seqs, kv, seed=seqs)


@pytest.mark.parametrize("D,P", [(64, 16), (128, 64)])
def test_one_row(wz, D, P):
    """Single tokens of heads that share nothing: one row a sequence and head."""
    run(wz, P, 16, 16, D, [1] * 9, [1, 2, 127, 128, 129, 0, 640, 4098, 1025], seed=D)


@pytest.mark.parametrize("tiles", [4, 5, 8, 9])
def test_whole_items_and_pieces(wz, tiles):
    """Tables of few tiles keep items whole, longer ones do not."""
    run(wz, 64, 2, 6, 128, [1, 1, 1], [128 * tiles, 0, 128 * tiles - 100])


def test_question_in_pieces(wz):
    """Few row tiles over many slots: pieces that the second kernel adds, some of them empty."""
    run(wz, 128, 1, 4, 64, [70, 5], [9000, 64])
    run(wz, 64, 1, 2, 96, [150], [5000], causal=False)


def test_more_tokens_than_said(wz):
    """max_new below a sequence's tokens is reported; nothing outside the arrays is touched."""
    P, D = 32, 64
    table, pages = tables([100], P, 3)
    gpu = ref.Cache(pages, 1, P, D, seed=6).on_gpu(wz)
    for n, max_new in ((20, 1), (300, 20)):
        room = torch.zeros((n + 4, 2, D), dtype=torch.bfloat16, device="cuda")
        q = torch.randn((n, 2, D), device="cuda").bfloat16()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        wz.wz_attend(q, gpu, i32(table), i32([0, n]), i32([100]), max_new=max_new, out=room[2:n + 2], device_status=status)
        assert int(status) == wz.STATUS_CACHE
        assert int(room[:2].abs().max()) == 0 and int(room[n + 2:].abs().max()) == 0


def test_replayed_from_a_graph(wz):
    """Append and attention captured in a CUDA graph: new inputs in the same buffers give what
    direct calls give."""
    P, heads, Hq, D = 64, 2, 8, 64
    g = torch.Generator().manual_seed(2)
    direct, captured = (ref.Cache(40, heads, P, D, seed=5).on_gpu(wz) for _ in range(2))
    table = i32([list(range(20)), list(range(20, 40))])
    cu, start, kv = i32([0, 1, 2]), i32([0, 0]), i32([0, 0])
    qkv = torch.zeros((2, Hq + 2 * heads, D), dtype=torch.bfloat16, device="cuda")
    rotation = wz.rotation_table(2000, D)
    ws = torch.empty(wz.wz_attend_workspace_size(2, Hq, D), dtype=torch.uint8, device="cuda")
    q, out = (torch.zeros((2, Hq, D), dtype=torch.bfloat16, device="cuda") for _ in range(2))

    def step(cache):
        wz.wz_kv_append(qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], cache, table, cu, start, max_new=1,
                        q=qkv[:, :Hq], q_out=q, rotation=rotation)
        wz.wz_attend(q, cache, table, cu, kv, max_new=1, out=out, workspace=ws)

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    start.copy_(i32([100, 1100]))
    kv.copy_(start + 1)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(wz.KvCache.empty(40, heads, P, D))
        torch.cuda.synchronize()
        with torch.cuda.graph(graph, stream=side):
            step(captured)
    for i in range(4):
        qkv.copy_(torch.randn(qkv.shape, generator=g))
        start.copy_(i32([100 + i, 1100 + i]))
        kv.copy_(start + 1)
        step(direct)
        want = out.clone()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)


def test_checked_build_agrees(wz):
    """The bounds-checked build reports nothing and gives the same bits, for both kernels and the
    append before them."""
    P, heads, Hq, D = 32, 2, 6, 96
    table, pages = tables([700, 333], P, 3)
    for new in ([1, 1], [40, 9]):
        start = [700 - new[0], 333 - new[1]]
        T = sum(new)
        qkv = torch.randn((T, Hq + 2 * heads, D), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        args = (i32(table), i32([0, new[0], T]))

        def both(status=None):
            gpu = ref.Cache(pages, heads, P, D, seed=6).on_gpu(wz)
            q = wz.wz_kv_append(qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], gpu, *args, i32(start), max_new=max(new),
                                q=qkv[:, :Hq], rotation=wz.rotation_table(800, D), device_status=status)
            out = wz.wz_attend(q, gpu, *args, i32([700, 333]), max_new=max(new), device_status=status)
            return q, gpu.k.view(torch.uint8), gpu.v.view(torch.uint8), gpu.k_scale, gpu.v_scale, out

        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        want = both()
        with wz.checked_library():
            got = both(status)
        assert int(status) == 0
        for a, b in zip(got, want):
            assert torch.equal(a, b)


def test_example_answers_from_the_cache(wz):
    """The example's outputs within the rounding of bf16 outputs and 8-bit weights of plain attention."""
    import importlib.util
    import os
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "answer_from_cache.py")
    spec = importlib.util.spec_from_file_location("answer_from_cache", path)
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    assert m.main() < 2.0 ** -7


@pytest.mark.parametrize("G,n", [(7, 10), (4, 32), (1, 128), (1, 17), (17, 1), (32, 4)])
def test_one_tile_of_rows(wz, G, n):
    """17 to 128 rows: both row tiles of a CTA hold them, in calls of few items; no slots, one tile,
    even and odd numbers of tiles, with and without splits."""
    for causal in (True, False):
        run(wz, 128, 1, G, 64, [n] * 5, [0, n, 129 + n, 257, 4000], causal=causal, seed=n)
    run(wz, 64, 8, 8 * G, 32, [n] * 30, [128 * (b % 9) + 7 * b + 1 for b in range(30)], seed=G)
    run(wz, 128, 8, 8 * G, 80, [n if b % 3 else max(1, n // 2) for b in range(45)], [b * 13 + 1 for b in range(45)], seed=G)
