"""The decoder cache's Python calls on the host, with stand-ins for tensors and for the library: what they refuse and
on which device they call."""

import contextlib

import pytest
import torch


@pytest.fixture(scope="module")
def wz():
    import paper_2607_23265_gb300.build as build
    build.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


class Fake:
    """What the binding reads of a CUDA tensor."""

    def __init__(self, *shape, dtype=torch.bfloat16, device=1, contiguous=True):
        self.shape, self.dtype, self._device, self._contiguous = torch.Size(shape), dtype, device, contiguous
        self.nbytes = dtype.itemsize * torch.Size(shape).numel()

    def stride(self):
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
        return 1 << 20


class Stream:
    cuda_stream = 0


def ints(*shape):
    return Fake(*shape, dtype=torch.int32)


@pytest.fixture
def call(wz, monkeypatch):
    """Runs one of the two calls with the cache on device 1 and device `current` current; the devices that the library
    was called on."""
    state = {"on": 0, "seen": []}

    class Library:
        def wz_attend(self, a):
            state["seen"].append(state["on"])
            return 0
        wz_kv_append = wz_attend

    @contextlib.contextmanager
    def device(index):
        saved, state["on"] = state["on"], index
        yield
        state["on"] = saved

    monkeypatch.setattr(wz, "_lib", Library())
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: state["on"], raising=False)
    cache = wz.KvCache.__new__(wz.KvCache)
    cache.index, cache.D, cache.heads, cache.page_tokens, cache.pages = 1, 64, 2, 64, 10
    cache._struct = wz.KvCacheStruct()

    def run(name, current=0, **kw):
        state["on"], state["seen"] = current, []
        cu, lens, table = ints(3), ints(2), ints(2, 8)
        if name == "attend":
            wz.wz_attend(Fake(2, 8, 64), cache, table, cu, lens, out=Fake(2, 8, 64), stream=Stream, **kw)
        else:
            wz.wz_kv_append(Fake(2, 2, 64), Fake(2, 2, 64), cache, table, cu, lens, stream=Stream, **kw)
        assert state["on"] == current
        return state["seen"]

    return run


@pytest.mark.parametrize("name", ["attend", "append"])
@pytest.mark.parametrize("current", [0, 1])
def test_the_cache_s_device_is_current_in_the_call(call, name, current):
    assert call(name, current) == [1]


@pytest.mark.parametrize("workspace", [Fake(1 << 26, dtype=torch.uint8, device=-1),
                                       Fake(1 << 26, dtype=torch.uint8, device=0),
                                       Fake(1 << 26, dtype=torch.uint8, contiguous=False)])
def test_workspaces_that_the_device_cannot_use(call, workspace):
    with pytest.raises(ValueError, match="workspace"):
        call("attend", workspace=workspace)
    assert call("attend", workspace=Fake(1 << 26, dtype=torch.uint8)) == [1]
