"""The decoder cache's entry points on the host: layouts, sizes, refusals.

Every call fails its checks, or has nothing to do, before any CUDA call."""

import ctypes as C

import pytest

P = 1 << 20   # aligned addresses that no call reads


@pytest.fixture(scope="module")
def wz():
    import paper_2607_23265_gb300.build as build
    build.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


def set_all(a, over):
    for k, v in over.items():
        if k.startswith("cache."):
            setattr(a.cache, k[6:], v)
        elif k == "section":
            a.section[:] = v
        else:
            setattr(a, k, v)
    return a


CACHE = {"cache.k": P, "cache.v": 2 * P, "cache.k_scale": 3 * P, "cache.v_scale": 4 * P, "cache.pages": 100,
         "cache.heads": 4, "cache.page_tokens": 64, "cache.D": 128}

CACHE_ERRORS = [
    ({"cache.k": None}, -1), ({"cache.v": None}, -1), ({"cache.k_scale": None}, -1), ({"cache.v_scale": None}, -1),
    ({"cache.k": P + 8}, -1), ({"cache.v": P + 4}, -1), ({"cache.v_scale": P + 2}, -1), ({"cache.pages": 0}, -1),
    ({"cache.pages": 1 << 31}, -2), ({"cache.pages": 1 << 30}, -2), ({"cache.heads": 0}, -1), ({"cache.heads": 1025}, -2),
    ({"cache.page_tokens": 48}, -1), ({"cache.page_tokens": 0}, -1), ({"cache.page_tokens": 256}, -1),
    ({"cache.D": 0}, -1), ({"cache.D": 72}, -2), ({"cache.D": 256}, -2),
]


def append_args(wz, **over):
    a = wz.KvAppendArgs()
    wz._lib.wz_kv_append_args_init(C.byref(a))
    assert (a.axes, a.max_new, a.rotation) == (1, 0, None)
    base = dict(CACHE, k=5 * P, v=6 * P, q=7 * P, q_out=8 * P, k_stride=512, v_stride=512, q_stride=3584,
                q_out_stride=3584, T=10, B=2, Hq=28, cu=9 * P, start=10 * P, page_table=11 * P, max_pages=8,
                rotation=12 * P, rotation_rows=100, rot=128)
    return set_all(a, {**base, **over})


@pytest.mark.parametrize("over,code", CACHE_ERRORS + [
    (dict(k=None), -1), (dict(v=None), -1), (dict(q_out=None), -1), (dict(k=5 * P + 8), -1), (dict(dtype=3), -1),
    (dict(T=-1), -1), (dict(T=1 << 31), -1), (dict(B=-1), -1), (dict(B=0), -1), (dict(B=1 << 25), -2),
    (dict(max_new=-1), -1), (dict(max_pages=0), -1), (dict(Hq=27), -1), (dict(Hq=0), -1), (dict(q=None), -1),
    (dict(k_stride=504), -1), (dict(v_stride=516), -1), (dict(q_stride=3576), -1), (dict(q_out_stride=0), -1),
    (dict(cu=None), -1), (dict(start=None), -1), (dict(page_table=None), -1), (dict(cu=9 * P + 2), -1),
    (dict(rotation=12 * P + 4), -1), (dict(rotation_rows=0), -1), (dict(rot=8), -1), (dict(rot=144), -1),
    (dict(rot=40), -1), (dict(axes=2), -1), (dict(axes=3), -1), (dict(axes=3, positions=P, section=[16, 24, 25]), -1),
    (dict(axes=3, positions=P, section=[-8, 48, 24]), -1), (dict(positions=P + 2), -1), (dict(device_status=P + 1), -1),
])
def test_append_refusals(wz, over, code):
    assert wz._lib.wz_kv_append(C.byref(append_args(wz, **over))) == code


def test_append_of_nothing(wz):
    assert wz._lib.wz_kv_append(C.byref(append_args(wz, T=0))) == 0
    assert wz._lib.wz_kv_append(None) == -1


def attend_args(wz, **over):
    a = wz.AttendArgs()
    wz._lib.wz_attend_args_init(C.byref(a))
    assert (a.causal, a.scale, a.lse) == (1, 0.0, None)
    base = dict(CACHE, q=5 * P, q_stride=3584, out=6 * P, out_stride=3584, T=10, B=2, Hq=28, cu=9 * P, kv_len=10 * P,
                page_table=11 * P, max_pages=8)
    return set_all(a, {**base, **over})


@pytest.mark.parametrize("over,code", CACHE_ERRORS + [
    (dict(q=None), -1), (dict(out=None), -1), (dict(q=5 * P + 4), -1), (dict(T=-1), -1), (dict(T=1 << 31), -1),
    (dict(B=0), -1), (dict(B=-1), -1), (dict(B=1 << 25), -2), (dict(Hq=0), -1), (dict(Hq=30), -1),
    (dict(max_new=-2), -1), (dict(max_pages=0), -1), (dict(q_stride=3000), -1), (dict(out_stride=3588), -1),
    (dict(cu=None), -1), (dict(kv_len=None), -1), (dict(page_table=None), -1), (dict(lse=P + 2), -1),
    (dict(device_status=P + 2), -1), (dict(scale=float("nan")), -1), (dict(scale=float("inf")), -1),
    (dict(workspace=12 * P, workspace_bytes=16), -5), (dict(workspace=12 * P + 64, workspace_bytes=1 << 40), -1),
])
def test_attend_refusals(wz, over, code):
    assert wz._lib.wz_attend(C.byref(attend_args(wz, **over))) == code


def test_attend_of_nothing(wz):
    assert wz._lib.wz_attend(C.byref(attend_args(wz, T=0))) == 0
    assert wz._lib.wz_attend(None) == -1


def test_workspace_size(wz):
    assert wz.wz_attend_workspace_size(1, 28, 128) > 0
    assert wz.wz_attend_workspace_size(-1, 28, 128) == 0
    assert wz.wz_attend_workspace_size(4, 0, 128) == 0


def test_struct_layouts_match_the_header(wz, tmp_path):
    """Sizes and the offsets of the last members, as a C compiler sees them."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include "wavezip.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu", '
                   "sizeof(wz_kv_cache), sizeof(wz_kv_append_args), offsetof(wz_kv_append_args, device_status), "
                   "sizeof(wz_attend_args), offsetof(wz_attend_args, workspace), offsetof(wz_kv_append_args, section)); "
                   "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert got == [C.sizeof(wz.KvCacheStruct), C.sizeof(wz.KvAppendArgs), wz.KvAppendArgs.device_status.offset,
                   C.sizeof(wz.AttendArgs), wz.AttendArgs.workspace.offset, wz.KvAppendArgs.section.offset]
