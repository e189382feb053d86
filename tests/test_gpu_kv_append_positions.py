"""A position outside the rotation table: the token's key and query are left out, its value and all others are not."""

import pytest
import torch

import kv_reference as ref
from test_gpu_kv_append import i32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


@pytest.mark.parametrize("form", ["slots", "one axis", "three axes"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_tokens_outside_the_table(wz, form, dtype):
    P, heads, Hq, D, rows, T, start = 64, 2, 6, 64, 150, 120, 40
    g = torch.Generator().manual_seed(3)
    qkv = torch.randn((T, Hq + 2 * heads, D), generator=g)
    positions = sections = None
    outside = torch.zeros(T, dtype=torch.bool)
    if form == "slots":
        outside[rows - start:] = True
    else:
        positions = torch.randint(0, rows, (T,) if form == "one axis" else (T, 3), generator=g, dtype=torch.int32)
        bad = [3, 23, 24, 77, 119]                      # the last two tokens of a page and the first of the next
        for i, x in enumerate(bad):
            place = (x,) if form == "one axis" else (x, (0, 2)[i % 2])
            positions[place] = (rows, -1, 2 ** 31 - 1, -2 ** 31, rows + 5)[i]
        outside[bad] = True
        if form == "three axes":
            sections = [20, 0, 12]
            positions[5, 1] = -7                        # an axis that no frequency takes concerns nothing
    qkv[outside] *= 1000                                # no say in their pages' scales
    qkv = qkv.to(dtype)
    dev = qkv.cuda()
    table = [[1, 2, 0]]
    host = ref.Cache(3, heads, P, D, seed=4)
    gpu = host.on_gpu(wz)
    before = gpu.k.view(torch.uint8).clone()
    q_out = torch.full((T, Hq, D), 7.0, dtype=dtype, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    rotation = wz.rotation_table(rows, D)
    wz.wz_kv_append(dev[:, Hq:Hq + heads], dev[:, Hq + heads:], gpu, i32(table), i32([0, T]), i32([start]),
                    q=dev[:, :Hq], q_out=q_out, rotation=rotation, sections=sections,
                    positions=None if positions is None else positions.cuda(), device_status=status)
    assert int(status) == wz.STATUS_CACHE

    # the reference with those tokens' keys all zeros at a sound position: they ask for no scale
    clean = qkv.clone()
    clean[outside, Hq:Hq + heads] = 0
    where = torch.arange(start, start + T, dtype=torch.int32) if positions is None else positions.clone()
    where = where.clamp(0, rows - 1)
    want, _ = ref.append(host, clean[:, Hq:Hq + heads], clean[:, Hq + heads:], table, [0, T], [start], rotation.cpu(), D,
                         False, where, sections, clean[:, :Hq], torch.float32)
    assert torch.equal(gpu.k_scale.cpu().double(), host.scale["k"])
    assert torch.equal(gpu.v_scale.cpu().double(), host.scale["v"])
    assert torch.equal(gpu.v.cpu().double(), host.codes["v"])
    left = torch.zeros((3, heads, P, D), dtype=torch.bool)
    for x in outside.nonzero()[:, 0].tolist():
        left[table[0][(start + x) // P], :, (start + x) % P] = True
    assert torch.equal(gpu.k.cpu().double()[~left], host.codes["k"][~left])
    assert torch.equal(gpu.k.view(torch.uint8).cpu()[left], before.cpu()[left])
    assert torch.equal(q_out.cpu()[~outside], want.to(dtype)[~outside])
    assert bool((q_out.cpu()[outside] == 7).all())
