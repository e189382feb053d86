"""wz_kv_append against a plain form: scales and older codes exactly, new numbers against 64 bits to
the rounding of their e4m3 code, and rotated queries and all codes to the bit against the documented
rounding (two products and their sum in f32, then the type's or the code's)."""

import pytest
import torch

import kv_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    assert torch.cuda.is_available()
    return m


def tables(lens, P, seed):
    """Rows of a page table for sequences of these lengths, pages in random order; the pool's size."""
    need = [-(-n // P) for n in lens]
    pool = torch.randperm(sum(need) + 2, generator=torch.Generator().manual_seed(seed)).tolist()
    width, rows, at = max(max(need), 1), [], 0
    for n in need:
        rows.append(pool[at:at + n] + [-1] * (width - n))
        at += n
    return rows, sum(need) + 2


def i32(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def check(cache, gpu, exact):
    """Scales equal; every code equal but new keys', which are within their own rounding of the exact
    number: half a step of the code, and the rotation's two products and sum in f32."""
    for name in "kv":
        codes = getattr(gpu, name).cpu().double()
        scale = getattr(gpu, name + "_scale").cpu().double()
        assert torch.equal(scale, cache.scale[name]), name
        fresh = torch.zeros(cache.shape, dtype=torch.bool)
        for n, page, row, part in exact:
            if n != name:
                continue
            fresh[page, :, row:row + part.shape[1]] = True
            s = scale[page][:, None, None]
            got = codes[page, :, row:row + part.shape[1]] * s
            half = torch.maximum(part.abs() * 2.0 ** -4, s * 2.0 ** -10)
            slack = part.abs().amax() * 2.0 ** -21
            inside = part.abs() <= 448 * s
            assert bool(((got - part).abs() <= half + slack)[inside].all()), name
            if name == "v":
                want = cache.codes[name][page, :, row:row + part.shape[1]]
                assert torch.equal(codes[page, :, row:row + part.shape[1]].nan_to_num(999), want.nan_to_num(999))
        assert torch.equal(codes[~fresh], cache.codes[name][~fresh]), name


CASES = [
    # page, heads, Hq, D, new, start, dtype, rot, interleaved, axes
    (16, 1, 1, 16, [1], [0], "bf16", 16, False, 1),
    (16, 2, 6, 80, [1, 0, 1, 1], [15, 3, 0, 31], "bf16", 80, False, 1),
    (64, 4, 28, 128, [1, 1, 1], [63, 64, 700], "bf16", 128, False, 3),
    (32, 2, 14, 128, [33, 5, 70], [31, 0, 17], "bf16", 128, True, 1),
    (128, 3, 3, 96, [257, 1], [100, 127], "bf16", 32, False, 3),
    (128, 1, 8, 128, [300], [1], "f32", 128, True, 3),
    (16, 16, 16, 64, [40, 0, 16, 17], [0, 9, 16, 8], "f32", 32, True, 1),
    (64, 2, 4, 48, [65, 64, 1, 2, 3, 100, 7], [0, 64, 63, 62, 62, 5, 57], "f32", 0, False, 1),
    (64, 2, 2, 112, [130], [0], "bf16", 112, False, 3),
]


@pytest.mark.parametrize("case", CASES, ids=[str(i) for i in range(len(CASES))])
def test_append(wz, case):
    P, heads, Hq, D, new, start, dtype, rot, interleaved, axes = case
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    g = torch.Generator().manual_seed(5 + P + D)
    T = sum(new)
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    table, pages = tables([a + b for a, b in zip(new, start)], P, 7)
    host = ref.Cache(pages, heads, P, D, seed=3)
    gpu = host.on_gpu(wz)
    qkv = torch.randn((T, Hq + 2 * heads, D), generator=g) * torch.exp2(torch.randint(-3, 4, (T, 1, 1), generator=g))
    qkv = qkv.to(dt)
    dev = qkv.cuda()
    sections = positions = rotation = None
    if rot:
        rotation = wz.rotation_table(1000, rot)
        if axes == 3:
            positions = torch.randint(0, 1000, (T, 3), generator=g, dtype=torch.int32)
            sections = [rot // 2 // 4 + 1, 3, rot // 2 - rot // 2 // 4 - 4]
    q_out = wz.wz_kv_append(dev[:, Hq:Hq + heads], dev[:, Hq + heads:], gpu, i32(table), i32(cu), i32(start),
                            max_new=max(new), q=dev[:, :Hq], rotation=rotation, interleaved=interleaved,
                            positions=None if positions is None else positions.cuda(), sections=sections)
    _, exact = ref.append(host, qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], table, cu, start,
                          None if rotation is None else rotation.cpu(), rot, interleaved, positions, sections)
    check(host, gpu, exact)
    stepwise = ref.Cache(pages, heads, P, D, seed=3)
    want, _ = ref.append(stepwise, qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], table, cu, start,
                         None if rotation is None else rotation.cpu(), rot, interleaved, positions, sections,
                         qkv[:, :Hq], torch.float32)
    assert torch.equal(q_out.cpu(), want.to(dt))
    for n in "kv":
        assert torch.equal(getattr(gpu, n).cpu().double(), stepwise.codes[n]), n
    # found through the lengths instead of through max_new: the same
    again = ref.Cache(pages, heads, P, D, seed=3).on_gpu(wz)
    wz.wz_kv_append(dev[:, Hq:Hq + heads], dev[:, Hq + heads:], again, i32(table), i32(cu), i32(start),
                    rotation=rotation, interleaved=interleaved,
                    positions=None if positions is None else positions.cuda(), sections=sections)
    for n in ("k", "v", "k_scale", "v_scale"):
        assert torch.equal(getattr(again, n).view(torch.uint8), getattr(gpu, n).view(torch.uint8)), n


def test_many_sequences_are_found(wz):
    """More sequences than one round of the search has places, with idle ones between."""
    P, heads, D = 16, 1, 32
    g = torch.Generator().manual_seed(1)
    new = [(0 if b % 3 == 1 else 1 + b % 21) for b in range(1300)]
    start = [(7 * b) % 40 for b in range(1300)]
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    table, pages = tables([a + b for a, b in zip(new, start)], P, 2)
    host = ref.Cache(pages, heads, P, D, seed=4)
    gpu = host.on_gpu(wz)
    kv = torch.randn((cu[-1], 2, D), generator=g).to(torch.bfloat16)
    dev = kv.cuda()
    wz.wz_kv_append(dev[:, :1], dev[:, 1:], gpu, i32(table), i32(cu), i32(start))
    _, exact = ref.append(host, kv[:, :1], kv[:, 1:], table, cu, start)
    check(host, gpu, exact)


def test_token_by_token_scales_grow(wz):
    """Single tokens of growing and shrinking size: the page's scale never falls until its row 0 is
    written again, and the codes are the reference's at every step."""
    P, heads, D = 32, 2, 64
    table = [[1, 0]]
    host = ref.Cache(3, heads, P, D, seed=9)
    gpu = host.on_gpu(wz)
    g = torch.Generator().manual_seed(8)
    for i in range(40):
        size = 2.0 ** ((i * 5) % 23 - 12)
        kv = (torch.randn((1, 2 * heads, D), generator=g) * size).to(torch.bfloat16)
        dev = kv.cuda()
        wz.wz_kv_append(dev[:, :heads], dev[:, heads:], gpu, i32(table), i32([0, 1]), i32([i]), max_new=1)
        _, exact = ref.append(host, kv[:, :heads], kv[:, heads:], table, [0, 1], [i])
        check(host, gpu, exact)
    assert torch.equal(gpu.k.cpu().double(), host.codes["k"])


def test_extremes(wz):
    """Zeros, numbers beyond both ends of the scales, infinities and NaN."""
    P, heads, D = 16, 1, 16
    x = torch.zeros((5, 2, D))
    x[0, 0, 3], x[0, 0, 4], x[0, 0, 5] = float("inf"), float("nan"), 3.0
    x[1, 0, 0], x[1, 0, 1] = float("-inf"), -448.0
    x[2, 1, :] = 1e30
    x[3, 1, 1] = 1e-38
    table = [[0]]
    host = ref.Cache(1, heads, P, D, seed=2)
    gpu = host.on_gpu(wz)
    dev = x.cuda()
    wz.wz_kv_append(dev[:, :1], dev[:, 1:], gpu, i32(table), i32([0, 5]), i32([0]))
    ref.append(host, x[:, :1], x[:, 1:], table, [0, 5], [0])
    for n in "kv":
        assert torch.equal(getattr(gpu, n + "_scale").cpu().double(), host.scale[n])
        assert torch.equal(getattr(gpu, n).cpu().double().nan_to_num(999), host.codes[n].nan_to_num(999)), n
    k = gpu.k.cpu().double()[0, 0]
    assert k[0, 3] == 448 and k[1, 0] == -448 and torch.isnan(k[0, 4])
    # nothing but zeros: the smallest scale
    gpu = host.on_gpu(wz)
    z = torch.zeros((1, 2, D), device="cuda")
    wz.wz_kv_append(z[:, :1], z[:, 1:], gpu, i32(table), i32([0, 1]), i32([0]))
    assert float(gpu.k_scale[0, 0]) == 2.0 ** ref.LOW and float(gpu.k.float()[0, 0, 0].abs().max()) == 0


def test_queries_in_place(wz):
    g = torch.Generator().manual_seed(3)
    x = torch.randn((9, 8, 64), generator=g).to(torch.bfloat16).cuda()
    cache = wz.KvCache.empty(2, 2, 16, 64)
    rotation = wz.rotation_table(64, 64)
    args = (i32([[1, 0]]), i32([0, 9]), i32([12]))
    want = wz.wz_kv_append(x[:, 4:6], x[:, 6:], cache, *args, q=x[:, :4], rotation=rotation)
    q = x[:, :4]
    wz.wz_kv_append(x[:, 4:6], x[:, 6:], cache, *args, q=q, q_out=q, rotation=rotation)
    assert torch.equal(q, want)


@pytest.mark.parametrize("what", ["page", "negative page", "table", "position", "start", "cu", "max_new"])
def test_entries_outside_are_reported(wz, what):
    """Contradicting entries set a status bit; what they do not concern is written, and nothing else."""
    P, heads, D = 16, 1, 32
    table, cu, start, max_new = [[0, 1], [2, 3]], [0, 3, 5], [0, 4], 0
    positions = torch.arange(5, dtype=torch.int32)
    if what == "page":
        table[0][0] = 5
    elif what == "negative page":
        table[0][0] = -1
    elif what == "table":
        start[0] = 32
    elif what == "position":
        positions[1] = 64
    elif what == "start":
        start[0] = -3
    elif what == "cu":
        cu = [0, 6, 5]
    elif what == "max_new":
        cu, max_new, start[0] = [0, 3, 30], 1, 0
    T = cu[-1]
    if what == "max_new":
        positions = torch.arange(T, dtype=torch.int32)
    x = torch.ones((T, 2, D), device="cuda")
    guard = wz.KvCache.empty(7, heads, P, D)      # pages 5 and 6 are past the cache that the call sees
    gpu = wz.KvCache(guard.k[:5], guard.v[:5], guard.k_scale[:5], guard.v_scale[:5])
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    wz.wz_kv_append(x[:, :1], x[:, 1:], gpu, i32(table), i32(cu), i32(start), max_new=max_new,
                    rotation=wz.rotation_table(64, 32), positions=positions.cuda(), device_status=status)
    assert int(status) == wz.STATUS_CACHE
    assert int(guard.v.view(torch.uint8)[4:].sum()) == 0
    if what in ("page", "negative page", "table", "start"):
        assert int(guard.v.view(torch.uint8)[:2].sum()) == 0
        assert bool((guard.v.float()[2, 0, 4:6] * guard.v_scale[2, 0] == 1).all())


def test_far_pages(wz):
    """A page whose first byte lies past 4 GiB."""
    P, heads, D = 128, 8, 128
    pages = (1 << 32) // (P * heads * D) + 3
    cache = wz.KvCache.empty(pages, heads, P, D)
    g = torch.Generator().manual_seed(3)
    x = torch.randn((130, 2 * heads, D), generator=g).to(torch.bfloat16).cuda()
    wz.wz_kv_append(x[:, :heads], x[:, heads:], cache, i32([[pages - 1, pages - 2]]), i32([0, 130]), i32([0]))
    got = cache.v[pages - 1].float() * cache.v_scale[pages - 1][:, None, None]
    want = x[:128, heads:].float().transpose(0, 1)
    assert bool(((got - want).abs() <= want.abs() * 2.0 ** -4 + cache.v_scale[pages - 1][:, None, None] * 2.0 ** -10).all())
    assert int(cache.v.view(torch.uint8)[:pages - 2].max()) == 0


def test_no_tokens(wz):
    cache = wz.KvCache.empty(1, 1, 16, 16)
    x = torch.empty((0, 2, 16), device="cuda")
    wz.wz_kv_append(x[:, :1], x[:, 1:], cache, i32([[0]]), i32([0, 0]), i32([0]))
    assert int(cache.k.view(torch.uint8).max()) == 0


def test_another_stream(wz):
    s = torch.cuda.Stream()
    cache = wz.KvCache.empty(1, 1, 16, 16)
    x = torch.ones((4, 2, 16), device="cuda")
    a = (i32([[0]]), i32([0, 4]), i32([0]))
    s.wait_stream(torch.cuda.current_stream())
    wz.wz_kv_append(x[:, :1], x[:, 1:], cache, *a, stream=s)
    s.synchronize()
    assert bool((cache.v.float()[0, 0, :4] * cache.v_scale[0, 0] == 1).all())
