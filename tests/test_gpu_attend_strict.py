"""wz_attend against 64 bits with each kernel's own tolerance, which no NaN and no infinity passes.

Per output channel, with p_t a row's weights (their sum 1) and v_t = s_t c_t a value as its page's scale times its code:

  weights      2^-8 + 2^-11 of sum p |v| for up to 16 rows a sequence and KV head: a weight is rounded to f16 (2^-11), then
               to two e4m3 numbers (each to 2^-4 of what it stands for).  The second number's last half step is 2^-10
               / 32 = 2^-15 beside a largest weight of 2^8 in its tile of 128 slots: 2^-23 max_tile(p s) sum_tile |c|.
               2^-11 of sum p |v| for more rows: f16.  Its last half step is 2^-25 beside a reference of 2^3 that is at
               most the largest: 2^-28 max(p s) sum |c|.
  sums         a step of the tensor cores adds 16 slots or more and loses at most 2^-20 of the absolute sum so far:
               kv 2^-24 sum p |v|
  logits       off by `off` (kv_reference.attend) and by their scales' and exponentials' rounding, 2^-17: weights and
               their sum off by exp(off + 2^-17) each
  output       rounded to bf16, whose numbers in [2^e, 2^(e+1)) are 2^(e-7) apart: half of that"""

import math

import pytest
import torch

import kv_reference as ref
import test_gpu_attend as cases
from test_gpu_kv_append import i32, tables

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wz():
    import __graft_entry__
    __graft_entry__.build()
    import paper_2607_23265_gb300.wavezip as m
    return m


def last_steps(host, q, table, cu, kv_len, causal, scale, few):
    """[T][Hq][D]: what the last half steps of the weights' formats can add up to, before the division by 2^23 or 2^28."""
    heads, P = host.shape[1:3]
    T, Hq, D = q.shape
    G = Hq // heads
    res = torch.zeros((T, Hq, D), dtype=torch.float64)
    for b in range(len(kv_len)):
        x0, n, kv = cu[b], cu[b + 1] - cu[b], kv_len[b]
        if not n or not kv:
            continue
        ids = torch.tensor(table[b][:-(-kv // P)])
        pad = -(-kv // 128) * 128 - kv
        for h in range(heads):
            K = (host.codes["k"][ids, h] * host.scale["k"][ids, h][:, None, None]).reshape(-1, D)[:kv]
            C = host.codes["v"][ids, h].reshape(-1, D)[:kv].abs()
            S = host.scale["v"][ids, h].repeat_interleave(P)[:kv]
            for i in range(n):
                see = min(kv, kv - n + i + 1) if causal else kv
                if see <= 0:
                    continue
                w = torch.softmax(q[x0 + i, h * G:(h + 1) * G].double() @ K[:see].T * scale, -1) * S[:see]
                if few:
                    top = torch.nn.functional.pad(w, (0, kv - see + pad)).view(G, -1, 128).amax(-1)
                    seen = torch.nn.functional.pad(C[:see], (0, 0, 0, kv - see + pad)).view(-1, 128, D).sum(1)
                    res[x0 + i, h * G:(h + 1) * G] = top @ seen
                else:
                    res[x0 + i, h * G:(h + 1) * G] = w.amax(-1)[:, None] * C[:see].sum(0)[None]
    return res


def run(wz, P, heads, Hq, D, new, kv_len, causal=True, seed=1, scale=None, gain=2.0, width=0):
    g = torch.Generator().manual_seed(seed)
    cu = [sum(new[:i]) for i in range(len(new) + 1)]
    table, pages = tables(kv_len, P, seed)
    host = ref.Cache(pages, heads, P, D, seed=seed)
    gpu = host.on_gpu(wz)
    cases.poison(gpu, table, kv_len, P)
    wide = [r + [-1] * (width - len(r)) for r in table]
    q = (torch.randn((cu[-1], Hq, D), generator=g) * gain).to(torch.bfloat16)
    lse = torch.full((cu[-1], Hq), 7.0, device="cuda")
    out = wz.wz_attend(q.cuda(), gpu, i32(wide), i32(cu), i32(kv_len), max_new=max(new), causal=causal, scale=scale, lse=lse)
    scale = 1 / math.sqrt(D) if scale is None else scale
    few = max(new) * (Hq // heads) <= 16
    want, wlse, mass, off = ref.attend(host, q, table, cu, kv_len, causal, scale)
    rel = (2.0 ** -8 + 2.0 ** -11 if few else 2.0 ** -11) + max(kv_len) * 2.0 ** -24
    rel = rel + torch.expm1(2 * (off[..., None] + 2.0 ** -17))
    err = rel * mass + last_steps(host, q, table, cu, kv_len, causal, scale, few) * 2.0 ** (-23 if few else -28)
    half_step = torch.exp2(torch.floor(torch.log2((want.abs() + err).clamp(min=2.0 ** -100))) - 8)
    tol = err + half_step + 1e-30
    diff = (out.cpu().double() - want).abs()
    assert bool((diff <= tol).all()), (float((diff / tol).nan_to_num(math.inf).max()), int((~(diff <= tol)).sum()))
    empty = torch.isneginf(wlse)
    assert torch.equal(torch.isneginf(lse.cpu()), empty) and bool((out.cpu()[empty] == 0).all())
    gap = (lse.cpu().double() - wlse).abs()[~empty]
    assert bool((gap <= (off + 2.0 ** -20 * wlse.abs() + 2.0 ** -19)[~empty]).all())


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", cases.FEW, ids=[str(i) for i in range(len(cases.FEW))])
def test_few_rows(wz, case, causal):
    run(wz, *case, causal=causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("case", cases.MANY, ids=[str(i) for i in range(len(cases.MANY))])
def test_many_rows(wz, case, causal):
    run(wz, *case, causal=causal)


@pytest.mark.parametrize("P,D", [(16, 16), (32, 80), (64, 112), (128, 128)])
def test_ends_inside_tiles(wz, P, D):
    """Lengths around a page's and a tile's end, unseen slots holding NaN, in every variant."""
    kv = [1, P - 1, P, P + 1, 127, 128, 129, 255, 257, 640]
    run(wz, P, 2, 2, D, [1] * 10, kv)
    run(wz, P, 2, 12, D, [1] * 10, kv)
    run(wz, P, 1, 8, D, [2] * 10, kv)
    run(wz, P, 1, 5, D, [9] * 10, kv)
    run(wz, P, 1, 2, D, [140, 1, 70, 3, 140, 140, 2, 140, 140, 30], kv)


def test_pieces(wz):
    run(wz, 128, 1, 2, 64, [1], [128 * 90 + 5])
    run(wz, 128, 1, 12, 64, [1], [128 * 90 + 127])
    run(wz, 128, 1, 4, 64, [70, 5], [9000, 64])
    run(wz, 64, 1, 2, 96, [150], [5000], causal=False)
    run(wz, 128, 1, 1, 80, [128] * 5, [0, 128, 257, 300, 4000])


@pytest.mark.parametrize("new,Hq", [(1, 2), (1, 14), (3, 10), (20, 6), (200, 2)])
def test_tables_far_wider_than_the_sequences(wz, new, Hq):
    """A table with room for 300,000 slots behind sequences of a few hundred: other plans, the same answers."""
    for P, seqs in ((16, 2), (128, 20)):
        kv = [1 + (97 * b + 250) % 900 for b in range(seqs)]
        run(wz, P, 2, Hq, 64, [new] * seqs, kv, width=300000 // P)


def test_equal_calls_give_equal_bits(wz):
    """Every plan, twenty times each on one workspace that holds something else every time."""
    for new, Hq, kv, width in ((1, 28, 741, 0), (1, 16, 20003, 0), (4, 16, 6000, 0), (10, 28, 9001, 0), (333, 28, 3000, 0),
                               (1, 4, 300, 9000)):
        table, pages = tables([kv], 64, 3)
        gpu = ref.Cache(pages, 4, 64, 128, seed=6).on_gpu(wz)
        q = torch.randn((new, Hq, 128), generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
        t, cu, n = i32([table[0] + [-1] * (width - len(table[0]))]), i32([0, new]), i32([kv])
        ws = torch.zeros(wz.wz_attend_workspace_size(new, Hq, 128), dtype=torch.uint8, device="cuda")
        want = wz.wz_attend(q, gpu, t, cu, n, workspace=ws).clone()
        for i in range(20):
            ws.fill_((37 * i + 5) % 256)
            assert torch.equal(wz.wz_attend(q, gpu, t, cu, n, workspace=ws), want)
