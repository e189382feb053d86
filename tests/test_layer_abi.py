"""The layer's matrix products on the host: layouts, sizes, refusals.

Every call fails its checks, or has nothing to do, before any CUDA call."""

import ctypes as C
import os
import subprocess

import pytest

P = 1 << 20   # aligned addresses that no call reads

CALLS = {
    "wz_linear": ("LinearArgs", dict(x=P, w=2 * P, bias=3 * P, residual=4 * P, out=5 * P, pre=6 * P, x_stride=64,
                                     w_stride=64, residual_stride=128, out_stride=128, pre_stride=128)),
    "wz_linear_backward": ("LinearBackwardArgs", dict(
        dy=P, x=2 * P, w=3 * P, bias=4 * P, pre=5 * P, dx=6 * P, dw=7 * P, db=8 * P, dy_stride=128, x_stride=64,
        w_stride=64, pre_stride=128, dx_stride=64, dw_stride=64, workspace=9 * P, workspace_bytes=1 << 30)),
    "wz_gated": ("GatedArgs", dict(x=P, w_gate=2 * P, w_up=3 * P, b_gate=4 * P, b_up=5 * P, out=6 * P, gate=7 * P,
                                   up=8 * P, x_stride=64, w_gate_stride=64, w_up_stride=64, out_stride=128,
                                   gate_stride=128, up_stride=128)),
    "wz_gated_backward": ("GatedBackwardArgs", dict(
        dout=P, x=2 * P, w_gate=3 * P, w_up=4 * P, b_gate=5 * P, b_up=6 * P, gate=7 * P, up=8 * P, dx=9 * P,
        dw_gate=10 * P, dw_up=11 * P, db_gate=12 * P, db_up=13 * P, dout_stride=128, x_stride=64, w_gate_stride=64,
        w_up_stride=64, gate_stride=128, up_stride=128, dx_stride=64, dw_gate_stride=64, dw_up_stride=64,
        workspace=14 * P, workspace_bytes=1 << 30)),
}


@pytest.fixture(scope="module")
def wz():
    import paper_2607_23265_gb300.build as build
    build.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


def call(wz, name, **over):
    struct, base = CALLS[name]
    a = getattr(wz, struct)()
    getattr(wz._lib, name + "_args_init")(C.byref(a))
    for k, v in {**base, "M": 10, "N": 128, "K": 64, **over}.items():
        setattr(a, k, v)
    return getattr(wz._lib, name)(C.byref(a))


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("over,code", [
    (dict(M=-1), -1), (dict(N=0), -1), (dict(K=0), -1), (dict(N=-8), -1), (dict(act=4), -1), (dict(act=-1), -1),
    (dict(M=(1 << 31) - 512), -2), (dict(N=65537), -2), (dict(K=65537), -2), (dict(M=1 << 30, N=2048), -2),
    (dict(M=1 << 30, K=2048), -2), (dict(device_status=P + 2), -1), (dict(x=None), -1), (dict(x=P + 8), -1),
    (dict(x_stride=56), -1), (dict(x_stride=68), -1), (dict(x_stride=0), -1), (dict(x_stride=-64), -1),
])
def test_refusals_of_all(wz, name, over, code):
    assert call(wz, name, **over) == code


REFUSED = {
    "wz_linear": [dict(w=None), dict(w=2 * P + 2), dict(w_stride=60), dict(out=None), dict(out=5 * P + 4), dict(out_stride=120),
                  dict(out_stride=130), dict(residual=4 * P + 8), dict(residual_stride=0), dict(pre=6 * P + 2),
                  dict(pre_stride=120), dict(bias=3 * P + 2)],
    "wz_linear_backward": [dict(dy=None), dict(dy=P + 8), dict(dy_stride=120), dict(w=None), dict(w_stride=0),
                           dict(pre=5 * P + 8), dict(pre_stride=4), dict(dx=6 * P + 2), dict(dx_stride=60),
                           dict(dw=7 * P + 2), dict(dw_stride=0), dict(db=8 * P + 2), dict(bias=4 * P + 1),
                           dict(workspace=9 * P + 64)],
    "wz_gated": [dict(w_gate=None), dict(w_up=None), dict(w_up=3 * P + 2), dict(w_gate_stride=60), dict(w_up_stride=0),
                 dict(out=None), dict(out_stride=120), dict(gate=None), dict(up=None), dict(gate=7 * P + 2),
                 dict(gate_stride=120), dict(up_stride=4), dict(b_gate=4 * P + 2), dict(b_up=5 * P + 1)],
    "wz_gated_backward": [dict(dout=None), dict(dout_stride=0), dict(w_gate=None), dict(w_up=None), dict(w_up_stride=60),
                          dict(gate=None), dict(up=None), dict(up=8 * P + 2), dict(gate_stride=4), dict(dx=9 * P + 2),
                          dict(dx_stride=60), dict(dw_gate=None), dict(dw_up=None), dict(dw_up=11 * P + 4),
                          dict(dw_gate_stride=0), dict(db_gate=12 * P + 2), dict(db_up=13 * P + 1),
                          dict(b_gate=5 * P + 3), dict(workspace=14 * P + 128)],
}


@pytest.mark.parametrize("name,over", [(n, o) for n, os_ in REFUSED.items() for o in os_])
def test_refusals_of_each(wz, name, over):
    assert call(wz, name, **over) == -1


@pytest.mark.parametrize("name", ["wz_linear_backward", "wz_gated_backward"])
def test_a_workspace_that_is_too_small(wz, name):
    need = getattr(wz, name + "_workspace_size")(10, 64, 128)
    assert need > 0
    assert call(wz, name, workspace_bytes=0) == -5
    assert call(wz, name, workspace_bytes=need // 2) == -5


@pytest.mark.parametrize("name", CALLS)
def test_null(wz, name):
    assert getattr(wz._lib, name)(None) == -1
    getattr(wz._lib, name + "_args_init")(None)


def test_no_rows(wz):
    """No row needs no address; the gradients of weights, where they are asked for, do."""
    nothing = dict(M=0, x=None, w=None, out=None, residual=None, pre=None)
    assert call(wz, "wz_linear", **nothing) == 0
    assert call(wz, "wz_gated", M=0, x=None, w_gate=None, w_up=None, out=None, gate=None, up=None) == 0
    none = dict(M=0, dy=None, x=None, w=None, pre=None, dx=None, dw=None, db=None)
    assert call(wz, "wz_linear_backward", **none, workspace=None) == 0
    assert call(wz, "wz_linear_backward", **{**none, "dw": 7 * P + 2}) == -1
    assert call(wz, "wz_gated", M=0, gate=None) == -1     # what goes together does so without rows too
    assert call(wz, "wz_gated_backward", M=0, dw_up=None) == -1


def test_init_fills_in_the_block_s_activation(wz):
    for struct, name, act in (("LinearArgs", "wz_linear", 0), ("LinearBackwardArgs", "wz_linear_backward", 0),
                              ("GatedArgs", "wz_gated", 3), ("GatedBackwardArgs", "wz_gated_backward", 3)):
        a = getattr(wz, struct)()
        a.M, a.act, a.x = 7, 9, P
        getattr(wz._lib, name + "_args_init")(C.byref(a))
        assert (a.M, a.act, a.x) == (0, act, None)


def test_workspace_sizes(wz):
    for f in (wz.wz_linear_backward_workspace_size, wz.wz_gated_backward_workspace_size):
        assert f(-1, 64, 64) == 0 and f(1, 0, 64) == 0 and f(1, 64, 65537) == 0 and f(1 << 31, 64, 64) == 0
        assert 0 < f(1, 64, 64) < f(1000, 64, 64) < f(100000, 64, 64)
        assert f(0, 64, 64) >= 0 and f(0, 65536, 65536) < 1 << 30
    # d, once or twice, an eighth of it for sums over 16 rows in fp32, and at most 48 MB of shares' sums
    for f, both in ((wz.wz_linear_backward_workspace_size, 1), (wz.wz_gated_backward_workspace_size, 2)):
        d = 18662 * 3584 * 2
        assert both * d <= f(18662, 3584, 3584) <= both * (d + d // 8 + 40 * 3584 * 4) + (48 << 20)
    assert wz.wz_gated_backward_workspace_size(4103, 3584, 14336) >= 2 * 4103 * 14336 * 2


def test_struct_layouts_match_the_header(wz, tmp_path):
    """Sizes and the offsets of every member, as a C compiler sees them."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    names = [(name, struct) for name, (struct, _) in CALLS.items()]
    prints = ""
    want = []
    for name, struct in names:
        s = getattr(wz, struct)
        prints += f'printf("%zu\\n", sizeof({name}_args));\n'
        want.append(C.sizeof(s))
        for field, _ in s._fields_:
            prints += f'printf("%zu\\n", offsetof({name}_args, {field}));\n'
            want.append(getattr(s, field).offset)
    src = tmp_path / "layout.c"
    src.write_text('#include <stddef.h>\n#include <stdio.h>\n#include "wavezip.h"\nint main(void) {\n' + prints + "return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.join(root, "include"), str(src), "-o", str(exe)], check=True)
    got = [int(x) for x in subprocess.run([str(exe)], capture_output=True, text=True).stdout.split()]
    assert got == want
