"""A CTA leaves when the last phase of each of its barriers is over.  Tiles a pair of SMs takes: one to five, so that either
tensor-memory buffer is the last one and has been used an even or an odd number of times; steps of K: fewer and more than
stages, whose last ones were used an even or an odd number of times.  A wait for a phase that does not come would say so."""

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
    with wz.checked_library():
        yield wz._lib.wz_check_mm_plan
        wz._lib.wz_check_mm_plan(0, 1, 64)


class Calls:
    def __init__(self, wz, M, N, K):
        self.wz, self.status = wz, torch.zeros(1, dtype=torch.int32, device="cuda")
        g = torch.Generator(device="cuda").manual_seed(M + N + K)
        self.x, self.w, self.u = (ref.random_rows(n, K, s, g) for n, s in ((M, 1.0), (N, K ** -0.5), (N, K ** -0.5)))
        self.dy = ref.random_rows(M, N, 0.1, g)

    def check(self):
        wz, kw = self.wz, dict(device_status=self.status)
        # one after the other: a CTA's memory is the next call's as soon as it has left
        got = [(wz.wz_linear(self.x, self.w, act="silu", **kw), wz.wz_gated(self.x, self.w, self.u, **kw)) for _ in range(6)]
        dx = [wz.wz_linear_backward(self.dy, self.x, self.w, need_w=False, **kw)[0] for _ in range(3)]
        db = [wz.wz_gated_backward(self.dy, self.x, self.w, self.u, need_x=False, need_w=False, need_b=True, **kw)[3:]
              for _ in range(3)]
        torch.cuda.synchronize()
        assert int(self.status) == 0
        for y, h in got[1:]:
            assert torch.equal(y, got[0][0]) and torch.equal(h, got[0][1])
        ref.check(got[0][0], ref.linear(self.x, self.w, None, "silu", None)[0], "y")
        ref.check(got[0][1], ref.gated(self.x, self.w, self.u, None, None, "silu")[0], "h")
        ref.check(dx[0], ref.gradients(self.x, [ref.linear_delta(self.dy, self.x, self.w, None, None, "none")], [self.w],
                                       True)[0], "dx")
        want = ref.gradients(self.x, ref.gated_delta(self.dy, self.x, self.w, self.u, None, None, None, None, "silu"),
                             [self.w, self.u])[2]
        ref.check(db[0][0], want[0], "db_gate")
        ref.check(db[0][1], want[1], "db_up")
        assert all(torch.equal(d, dx[0]) for d in dx) and all(torch.equal(a, b) for d in db for a, b in zip(d, db[0]))


@pytest.mark.parametrize("steps", [1, 5, 6, 7, 13])
@pytest.mark.parametrize("tiles", [1, 77, 153, 229, 305])
def test_tiles_of_a_pair(wz, forced, tiles, steps):
    forced(1, 1, 64)
    Calls(wz, 256 * tiles - 3, 250, 64 * steps - 1).check()


@pytest.mark.parametrize("steps", [2, 3, 8, 9, 11, 12, 13, 25, 37])
@pytest.mark.parametrize("plan", [(2, 1, 64), (2, 2, 128), (3, 1, 96), (3, 2, 256), (3, 3, 64), (3, 4, 32)])
def test_stages_of_few_tiles(wz, forced, plan, steps):
    forced(*plan)
    Calls(wz, 300, 520, 64 * steps).check()
