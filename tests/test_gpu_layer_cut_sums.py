"""Products of more than 4,096 terms that are formed again for their slopes are two sums or more, each half as long or less.

A tensor core adds 16 products and the sum so far at a time: it lines them up below the largest of them, cuts each off,
towards 0, two bits behind the 24 of a sum, and cuts what they make to 24 bits again.  (Found by comparing sums of 128 to
4,096 terms with such models, all of whose bits are equal.)  That is done here in 64 bits for one sum and for two, of
the even and of the odd steps of 64; with terms of one sign nothing evens out, and one sum loses twice what two lose, or
more.  What a call loses has to be below the middle between them.

It is read from bias gradients of a single row, which are f32.  Behind a gated product without activation they are
dy u and dy g: the sums themselves.  Behind SiLU they are its slope, from whose difference the sum's follows:
the slope is off by 2^-22 or so by itself, which with a derivative of 0.3 is 1e-6 of a sum around 1, on either side."""

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


def cut(v, exponent, bits):
    """v without what is behind `bits` bits of a number with this exponent."""
    grid = torch.ldexp(torch.ones_like(v), exponent - bits)
    return torch.trunc(v / grid) * grid


def lost(x, w, sums):
    """What x w^T in `sums` sums loses, relative, on average over the outputs."""
    terms = w.double() * x.double()
    pieces = torch.nn.functional.pad(terms, (0, -terms.shape[1] % 16)).view(terms.shape[0], -1, 16)
    s = torch.zeros((sums, terms.shape[0]), dtype=torch.float64, device=x.device)
    for i in range(pieces.shape[1]):
        which = i // 4 % sums
        parts = torch.cat([pieces[:, i], s[which][:, None]], 1)
        largest = torch.frexp(parts.abs().max(1, keepdim=True).values).exponent
        total = cut(parts, largest.expand_as(parts), 26).sum(1)
        s[which] = cut(total, torch.frexp(total).exponent, 24)
    exact = terms.sum(1)
    return float(((exact - s.sum(0)) / exact).mean())


@pytest.mark.parametrize("plan", [(0, 1, 64), (1, 1, 64), (2, 4, 16), (3, 4, 32)])
@pytest.mark.parametrize("M,row", [(1, 0), (300, 217)])
@pytest.mark.parametrize("K", [4224, 14336])
def test_long_sums_are_shared(wz, forced, K, M, row, plan):
    forced(*plan)
    N = 264
    g = torch.Generator(device="cuda").manual_seed(K + M)

    def half(n, gain):
        t = ((0.5 + 0.5 * torch.rand((n, K), generator=g, device="cuda"))).bfloat16()
        return t * gain   # a power of 2

    x, wg, wu = half(M, 1.0), half(N, 2.0 ** -13), half(N, 2.0 ** -13)
    dy = torch.zeros((M, N), dtype=torch.bfloat16, device="cuda")
    dy[row] = 1.0
    kw = dict(need_x=False, need_w=False, need_b=True)
    g64, u64 = x[row].double() @ wg.double().T, x[row].double() @ wu.double().T
    one, two = (lost(x[row], wg, n) for n in (1, 2))
    assert one > 2 * two and one > 1e-5
    found = {}
    _, _, _, db_gate, db_up = wz.wz_gated_backward(dy, x, wg, wu, act="none", **kw)
    found["u"], found["g"] = ((u64 - db_gate.double()) / u64).mean(), ((g64 - db_up.double()) / g64).mean()
    # SiLU's slope where its derivative is steep: the sums shifted to around 1 by the bias
    bias = (1.0 - g64).float()
    at = g64 + bias.double()
    s = torch.sigmoid(at)
    steep = s * (1 - s) * (2 + at * (1 - 2 * s))
    db = wz.wz_linear_backward(dy, x, wg, act="silu", bias=bias, **kw)[2]
    found["p"] = ((ref.slope(at, "silu") - db.double()) / steep / g64).mean()
    found = {k: float(v) for k, v in found.items()}
    print(f"{K} {M} {plan}: one {one:.2e} two {two:.2e} found", {k: f"{v:.2e}" for k, v in found.items()})
    for name, off in found.items():
        assert -1e-6 < off < (one + two) / 2 + (1e-6 if name == "p" else 0), (name, off, one, two)
