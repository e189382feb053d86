"""Performance cases of the decoder cache: what a user does with condensed tokens after the projector.

listed()            the named cases
draw(rng)           one more case of the same ranges
prepare(case, seed) inputs, caches and tables on the GPU
run(state)          one pass through an operator, and its outputs
work(case)          bytes and flops of one pass that no implementation can do without
exact(case, seed)   the outputs in 64 bits, from torch alone

Two operators over one paged cache of keys and values.  A page holds P tokens of every KV
head in e4m3 (8 bits) and, for each head, one power-of-two scale for its keys and one for its
values; a sequence's pages are listed in its row of a table.

  append   wz_kv_append: new tokens' keys (rotated by position) and values into the cache, the
           queries rotated beside them.  A page's scale grows when a new token needs it, and the
           tokens that the page held are expressed in the new scale.
  attend   wz_attend: softmax attention of the queries over the cache, with log-sum-exp

`own` chooses the side that run() computes: the plain form (elementary torch operations in 32
bits) or the library's calls.  Lengths follow from the case alone, contents from the seed.
"""

import math

import torch

own = False

MOST_NEW = 18699        # the 18,662 condensed tokens of a 256-frame 27 x 27 video at ratio 0.1, and a question
E4M3_MAX = 448.0
LOW, HIGH = -60, 60     # exponents of a page's scale


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _append(name, **kw):
    case = {"name": name, "op": "append", "B": 1, "new": 1, "past": 0, "ragged": False, "Hq": 28, "Hkv": 4, "D": 128,
            "page": 64, "dtype": "bf16", "axes": 1, "rot": 128, "interleaved": False}
    case.update(kw)
    return case


def _attend(name, **kw):
    case = {"name": name, "op": "attend", "B": 1, "new": 1, "past": 0, "ragged": False, "Hq": 28, "Hkv": 4, "D": 128,
            "page": 64, "causal": True}
    case.update(kw)
    return case


def listed():
    return [
        # one answer's next token after a condensed video: the smallest call, where latency counts
        _append("append_token", past=4103),
        # the next token of 64 answers at once, over pages of 32 tokens
        _append("append_token_64", B=64, past=18699, ragged=True, page=32),
        # the prompt of the 256-frame video with its question, at positions (t, i, j)
        _append("append_prompt_18699", new=MOST_NEW, axes=3),
        # 32 videos of a serving batch that end inside pages, fp32 projections, 64-wide heads, interleaved pairs
        _append("append_chunks_f32", B=32, new=577, past=2741, ragged=True, Hq=16, Hkv=16, D=64, page=16, dtype="f32",
                rot=32, interleaved=True),
        # one answer's next token over a short condensed clip: latency
        _attend("decode_741", past=740),
        # ... over hours of video: one sequence has to fill the whole GPU
        _attend("decode_200003", past=200002),
        # ... of 64 answers of very different lengths
        _attend("decode_64_ragged", B=64, past=MOST_NEW, ragged=True, page=32),
        # ungrouped heads of 64 channels in short pages
        _attend("decode_16_mha64", B=16, past=4097, ragged=True, Hq=16, Hkv=16, D=64, page=16),
        # a draft of four tokens checked for eight answers at once
        _attend("verify_8x4", B=8, new=4, past=16381, ragged=True, Hq=32, Hkv=8, page=128),
        # a question of 333 tokens on a long video that the cache holds
        _attend("question_333_on_18699", new=333, past=MOST_NEW),
        # prompts of four videos, each with nothing before it
        _attend("prompts_4x2741", B=4, new=2741, ragged=True, Hq=32, Hkv=8),
        # the largest: one prompt of 6,151 tokens
        _attend("prompt_6151", new=6151),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


HEADS = [(28, 4), (28, 4), (32, 8), (16, 16), (8, 1), (14, 2), (24, 3), (5, 5)]


def draw(rng):
    Hq, Hkv = rng.choice(HEADS)
    D = rng.choice([128, 128, 64, 96, 80])
    page = rng.choice([16, 32, 64, 128])
    B = _log_int(rng, 1, 64)
    ragged = rng.random() < 0.7
    common = {"B": B, "ragged": ragged, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page}
    if rng.random() < 0.35:
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = max(1, min(MOST_NEW // B, MOST_NEW * 36 * 128 // (B * (Hq + 2 * Hkv) * D * (2 if dtype == "f32" else 1))))
        new = 1 if rng.random() < 0.3 else _log_int(rng, 1, most)
        case = _append("", **common, new=new, past=_log_int(rng, 1, 20000) - 1, dtype=dtype, axes=rng.choice([1, 1, 3]),
                       rot=D if rng.random() < 0.7 else 32, interleaved=rng.random() < 0.3)
    else:
        kind = rng.choice(["decode", "decode", "few", "chunk", "prompt"])
        cap = 64 * MOST_NEW * 4 * 128 // (B * Hkv * D) // 2           # tokens a sequence: bytes of the largest decode
        if kind == "decode":
            new, past = 1, _log_int(rng, 1, max(1, min(200003, cap))) - 1
        elif kind == "few":
            new, past = rng.randint(2, 8), _log_int(rng, 1, max(1, min(60000, cap))) - 1
        else:
            pairs = 6151 * 6151 * 28 * 128 // 4 // (B * Hq * D)       # half of the largest prompt's products
            new = _log_int(rng, 9, max(10, min(6000, math.isqrt(pairs))))
            past = 0 if kind == "prompt" else _log_int(rng, 1, max(1, min(cap, pairs // new))) - 1
        case = _attend("", **common, new=new, past=past, causal=rng.random() < 0.85)
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# lengths and inputs
# ---------------------------------------------------------------------------

def _lengths(case):
    """New tokens and tokens cached before them, of each sequence."""
    B, new, past = case["B"], case["new"], case["past"]
    if not case["ragged"]:
        return [new] * B, [past] * B
    part = [((b + 1) * 0.6180339887498949) % 1.0 for b in range(B)]
    part[0] = 1.0                                                     # one sequence has the full lengths
    news = [max(1, int(new * (0.25 + 0.75 * f))) for f in part]
    if case["op"] == "append" and B > 3:
        news[2] = 0                                                   # an idle one
    return news, [int(past * (0.03 + 0.97 * f * f)) for f in part]


def _rotation(positions, rot):
    """[positions][rot] f32: the cosines of the rot / 2 angles, then the sines."""
    inv = 10000.0 ** (-torch.arange(0, rot // 2, dtype=torch.float64, device="cuda") * 2 / rot)
    ang = torch.arange(positions, dtype=torch.float64, device="cuda")[:, None] * inv
    return torch.cat([ang.cos(), ang.sin()], 1).float()


def _sections(rot):
    a = rot // 2 // 4
    b = (rot // 2 - a) // 2
    return [a, b, rot // 2 - a - b]


def prepare(case, seed):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    B, Hq, Hkv, D, P = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    news, pasts = _lengths(case)
    T = sum(news)
    totals = [n + p for n, p in zip(news, pasts)]
    need = [-(-t // P) for t in totals]
    used, pages, width = sum(need), sum(need) + 3, max(max(need), 1)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    cu = torch.zeros(B + 1, dtype=torch.int32, device=dev)
    cu[1:] = torch.cumsum(i32(news), 0)
    # a sequence's pages lie anywhere in the pool; what the table does not need is -1
    order = torch.randperm(pages, generator=g, device=dev).to(torch.int32)
    lens = i32(need)
    column = torch.arange(width, device=dev)
    valid = column[None, :] < lens[:, None]
    table = torch.full((B, width), -1, dtype=torch.int32, device=dev)
    table[valid] = order[:used]
    s = {"case": case, "cu": cu, "start": i32(pasts), "kv_len": i32(totals), "table": table, "T": T, "width": width}
    # keys with a few strong channels, values of about unit size; a page's scale fits its largest element
    shape = (pages, Hkv, P, D)
    boost = 1 + 5 * (torch.rand(D, generator=g, device=dev) < 0.05).float()
    full = case["op"] == "attend"
    for name, gain in (("k", boost), ("v", torch.ones_like(boost))):
        x = torch.randn(shape, generator=g, device=dev, dtype=torch.float32)
        x.mul_(gain)
        if full:
            e = _need(x.abs().amax((2, 3)))
        else:
            e = torch.full((pages, Hkv), -6 if name == "v" else -4, dtype=torch.int32, device=dev)
        scale = torch.exp2(e.float())
        s[name + "_cache"] = (x / scale[:, :, None, None]).clamp_(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        s[name + "_scale"] = scale
        del x
    if full:
        # memory that no token was written to holds anything, NaN included
        free = order[used:].long()
        last = torch.tensor([t % P for t in totals], device=dev)
        at = table.gather(1, (lens.long() - 1).clamp(min=0)[:, None]).long()[:, 0]
        stale = (torch.arange(P, device=dev)[None, :] >= last[:, None]) & (last > 0)[:, None] & (lens > 0)[:, None]
        seq, row = stale.nonzero(as_tuple=True)
        for name in ("k_cache", "v_cache"):
            bits = s[name].view(torch.uint8)
            bits[at[seq], :, row] = 0x7F
            bits[free] = 0x7F
    dt = torch.float32 if case.get("dtype") == "f32" else torch.bfloat16
    # queries, keys and values are slices of one projection's rows
    qkv = torch.randn((T, Hq + 2 * Hkv, D), generator=g, device=dev)
    qkv[:, Hq:Hq + Hkv].mul_(boost)
    qkv[:, :Hq].mul_(2)                                       # attention logits of a few units
    qkv = qkv.to(dt)
    s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
    if case["op"] == "append":
        s["positions"], s["sections"] = None, None
        most = max(totals)
        if case["axes"] == 3:
            # frame and grid place of each condensed token; a question's tokens have all three alike
            x = torch.arange(T, device=dev)
            s["positions"] = torch.stack([x // 73, x % 73 // 9, x % 9], 1).to(torch.int32)
            s["positions"][-max(1, T // 500):] = (x[-max(1, T // 500):, None] // 73).to(torch.int32)
            s["sections"] = _sections(case["rot"])
            most = T // 73 + 74
        s["rotation"] = _rotation(most, case["rot"])
        s["q_out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
    else:
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
        s["lse"] = torch.empty((T, Hq), dtype=torch.float32, device=dev)
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

def _need(amax):
    """The smallest n with amax <= 448 * 2^n, in [LOW, HIGH] (0: LOW)."""
    m, e = torch.frexp(amax)
    n = torch.where(m <= 0.875, e - 9, e - 8)
    return torch.where(amax > 0, n, torch.full_like(n, LOW)).clamp(LOW, HIGH)


def _rotate(x, c, s, rot, interleaved):
    """The first `rot` channels of x [T][H][D] by the angles of c, s [T][rot / 2], in f32."""
    x = x.float()
    c, s = c[:, None, :], s[:, None, :]
    if interleaved:
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = x[..., :rot // 2], x[..., rot // 2:rot]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_append(st):
    case, cu, start, table, T = st["case"], st["cu"].long(), st["start"].long(), st["table"], st["T"]
    P, rot = case["page"], case["rot"]
    x = torch.arange(T, device=cu.device)
    seq = torch.searchsorted(cu, x, right=True) - 1
    slot = start[seq] + x - cu[seq]
    page, row = table[seq, slot // P].long(), slot % P
    tab, half = st["rotation"], rot // 2
    if st["positions"] is None:
        c, s = tab[slot, :half], tab[slot, half:]
    else:
        f = torch.arange(half, device=cu.device)
        axis = (f >= st["sections"][0]).long() + (f >= st["sections"][0] + st["sections"][1]).long()
        pos = st["positions"].long()[:, axis]
        c, s = tab[pos, f], tab[pos, f + half]
    q = _rotate(st["q"], c, s, rot, case["interleaved"])
    st["q_out"].copy_(q)
    first = table.gather(1, (start // P)[:, None].clamp(max=table.shape[1] - 1))[:, 0].long()
    partial = (start % P > 0) & (cu[1:] > cu[:-1])
    first = torch.where(partial, first, torch.zeros_like(first))
    older = partial[:, None] & (torch.arange(P, device=cu.device)[None, :] < (start % P)[:, None])
    for name, new in (("k", _rotate(st["k"], c, s, rot, case["interleaved"])), ("v", st["v"].float())):
        cache, scale = st[name + "_cache"], st[name + "_scale"]
        finite = torch.where(torch.isfinite(new), new.abs(), torch.zeros_like(new))
        need = _need(finite.amax(-1)).to(torch.int32)
        at = page[:, None].expand_as(need).long()
        most = torch.full_like(scale, LOW, dtype=torch.int32).scatter_reduce(0, at, need, "amax")
        touched = torch.zeros_like(scale, dtype=torch.bool).index_fill(0, page, True)
        fresh = torch.zeros_like(scale, dtype=torch.int32).scatter_reduce(
            0, at, (row == 0).int()[:, None].expand_as(need), "amax") > 0
        fit = torch.exp2(most.float())
        grown = torch.where(touched, torch.where(fresh, fit, torch.maximum(scale, fit)), scale)
        # the tokens that a sequence's first page holds already, in the page's new scale
        old = cache[first].float() * (scale[first] / grown[first])[:, :, None, None]
        old = old.clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        b, r = older.nonzero(as_tuple=True)
        bits = cache.view(torch.uint8)
        bits[first[b], :, r] = old.view(torch.uint8)[b, :, r]
        put = (new / grown[page][:, :, None]).clamp(-E4M3_MAX, E4M3_MAX).to(torch.float8_e4m3fn)
        bits[page, :, row] = put.view(torch.uint8)
        scale.copy_(grown)


def _plain_attend(st):
    case, cu, kv, table, T = st["case"], st["cu"].long(), st["kv_len"].long(), st["table"], st["T"]
    B, Hq, Hkv, D, P, new = (case[k] for k in ("B", "Hq", "Hkv", "D", "page", "new"))
    G, S, dev = Hq // Hkv, st["width"] * case["page"], cu.device
    pages = table.clamp(min=0).long()
    t = torch.arange(S, device=dev)
    held = t[None, :] < kv[:, None]                                            # [B][S]
    keys, values = ((st[n + "_cache"][pages].float() * st[n + "_scale"][pages][:, :, :, None, None])
                    .permute(0, 2, 1, 3, 4).reshape(B, Hkv, S, D) for n in "kv")
    values = torch.where(held[:, None, :, None], values, torch.zeros_like(values))
    x = torch.arange(T, device=dev)
    seq = torch.searchsorted(cu, x, right=True) - 1
    at = x - cu[seq]
    q = torch.zeros((B, new, Hq, D), device=dev)
    q[seq, at] = st["q"].float()
    q = q.reshape(B, new, Hkv, G, D).permute(0, 2, 3, 1, 4).reshape(B, Hkv, G * new, D)
    scores = torch.matmul(q, keys.transpose(2, 3)).mul_(st["scale"])           # [B][Hkv][G * new][S]
    n = kv[:, None].expand(B, new)
    if case["causal"]:
        n = n - (cu[1:] - cu[:-1])[:, None] + torch.arange(1, new + 1, device=dev)[None, :]
    seen = (t[None, None, :] < n[:, :, None]) & held[:, None, :]               # [B][new][S]
    scores = scores.view(B, Hkv, G, new, S)
    scores.masked_fill_(~seen[:, None, None], -math.inf)
    top = scores.amax(-1, keepdim=True)
    top = torch.where(torch.isneginf(top), torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    out = torch.matmul(p.view(B, Hkv, G * new, S), values).view(B, Hkv, G, new, D)
    out = out / torch.where(total > 0, total, torch.ones_like(total))
    lse = (top + total.log())[..., 0]
    st["out"].copy_(out.permute(0, 3, 1, 2, 4).reshape(B, new, Hq, D)[seq, at])
    st["lse"].copy_(lse.permute(0, 3, 1, 2).reshape(B, new, Hq)[seq, at])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _library(st):
    """The binding and the state's cache handle and workspace, which a serving program keeps."""
    if "wz" not in st:
        import paper_2607_23265_gb300.wavezip as wz
        st["wz"] = wz
        st["cache"] = wz.KvCache(st["k_cache"], st["v_cache"], st["k_scale"], st["v_scale"])
        if st["case"]["op"] == "attend":
            n = wz.wz_attend_workspace_size(st["T"], st["case"]["Hq"], st["case"]["D"])
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    return st["wz"]


def run(st):
    case = st["case"]
    if case["op"] == "append":
        if own:
            _library(st).wz_kv_append(st["k"], st["v"], st["cache"], st["table"], st["cu"], st["start"],
                                      max_new=case["new"], q=st["q"], q_out=st["q_out"], rotation=st["rotation"],
                                      positions=st["positions"], sections=st["sections"],
                                      interleaved=case["interleaved"])
        else:
            _plain_append(st)
        return [st["q_out"], st["k_cache"], st["k_scale"], st["v_cache"], st["v_scale"]]
    if own:
        _library(st).wz_attend(st["q"], st["cache"], st["table"], st["cu"], st["kv_len"], max_new=case["new"],
                               causal=case["causal"], scale=st["scale"], out=st["out"], lse=st["lse"],
                               workspace=st["workspace"])
    else:
        _plain_attend(st)
    return [st["out"], st["lse"]]


def work(case):
    B, Hq, Hkv, D, P = (case[k] for k in ("B", "Hq", "Hkv", "D", "page"))
    news, pasts = _lengths(case)
    T = sum(news)
    if case["op"] == "append":
        e = 4 if case["dtype"] == "f32" else 2
        rows = T if case["axes"] == 1 else T // 73 + 74
        blocks = sum(-(-(p + n) // P) - p // P for n, p in zip(news, pasts) if n)
        return {"bytes": T * (2 * Hq * D * e + 2 * Hkv * D * (e + 1)) + min(rows, T * case["axes"]) * case["rot"] * 4
                + T * (12 if case["axes"] == 3 else 0) + blocks * (Hkv * 16 + 4) + 8 * B,
                "flops": T * ((Hq + Hkv) * case["rot"] * 3 + 2 * Hkv * D * 2)}
    pairs = read = 0
    for n, p in zip(news, pasts):
        pairs += n * p + n * (n + 1) // 2 if case["causal"] else n * (n + p)
        read += n + p
    return {"bytes": read * Hkv * 2 * D + -(-read // P) * (8 * Hkv + 4) + T * Hq * (4 * D + 4) + 8 * B,
            "flops": 4 * D * Hq * pairs}


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _round_e4m3(y):
    """y (f64, |y| <= 448 or saturated) to the nearest e4m3 value, ties to even."""
    y = y.clamp(-E4M3_MAX, E4M3_MAX)
    e = torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6)))
    q = torch.exp2(e - 3)
    return torch.round(y / q) * q


def _exact_append(case, seed):
    st = prepare(case, seed)
    news, pasts = _lengths(case)
    P, rot, D = case["page"], case["rot"], case["D"]
    half = rot // 2
    tab = st["rotation"].double()
    table = st["table"].tolist()

    def turned(x, pos):                                       # x [n][H][D], pos [n][rot / 2] (a position a frequency)
        f = torch.arange(half, device=x.device)
        c, s = tab[pos, f][:, None], tab[pos, half + f][:, None]
        x = x.double().clone()
        lo = torch.arange(0, rot, 2, device=x.device) if case["interleaved"] else f
        hi = lo + (1 if case["interleaved"] else half)
        a, b = x[..., lo], x[..., hi]
        x[..., lo], x[..., hi] = a * c - b * s, a * s + b * c
        return x

    q_out = torch.empty(st["q_out"].shape, dtype=torch.float64, device="cuda")
    caches = {n: st[n + "_cache"].double() for n in "kv"}
    scales = {n: st[n + "_scale"].double().clone() for n in "kv"}
    x0 = 0
    for b, (n, past) in enumerate(zip(news, pasts)):
        if not n:
            continue
        x = slice(x0, x0 + n)
        x0 += n
        if st["positions"] is None:
            pos = torch.arange(past, past + n, device="cuda")[:, None].expand(n, half)
        else:
            a = st["sections"]
            pos = torch.repeat_interleave(st["positions"][x].long(), torch.tensor(a, device="cuda"), 1)
        q_out[x] = turned(st["q"][x], pos)
        fresh = {"k": turned(st["k"][x], pos), "v": st["v"][x].double()}
        for name, rows in fresh.items():
            cache, scale = caches[name], scales[name]
            for j in range(past // P, -(-(past + n) // P)):
                page = table[b][j]
                lo, hi = max(j * P, past), min((j + 1) * P, past + n)
                part = rows[lo - past:hi - past]              # [tokens][Hkv][D]
                top = part.abs().amax((0, 2))
                fit = torch.exp2(torch.ceil(torch.log2((top / E4M3_MAX).clamp(min=2.0 ** LOW, max=2.0 ** HIGH))))
                now = fit if lo == j * P else torch.maximum(scale[page], fit)
                held = lo - j * P
                if held:
                    cache[page, :, :held] = _round_e4m3(cache[page, :, :held] * (scale[page] / now)[:, None, None])
                cache[page, :, held:hi - j * P] = _round_e4m3(part / now[None, :, None]).transpose(0, 1)
                scale[page] = now
    return [q_out, caches["k"], scales["k"], caches["v"], scales["v"]]


def _exact_attend(case, seed):
    st = prepare(case, seed)
    news, pasts = _lengths(case)
    Hq, Hkv, D, P = (case[k] for k in ("Hq", "Hkv", "D", "page"))
    G = Hq // Hkv
    out = torch.zeros((st["T"], Hq, D), dtype=torch.float64, device="cuda")
    lse = torch.full((st["T"], Hq), -math.inf, dtype=torch.float64, device="cuda")
    x0 = 0
    for b, (n, past) in enumerate(zip(news, pasts)):
        kv, x = n + past, slice(x0, x0 + n)
        x0 += n
        if not n or not kv:
            continue
        ids = st["table"][b, :-(-kv // P)].long()
        for h in range(Hkv):
            K, V = ((st[c + "_cache"][ids, h].double() * st[c + "_scale"][ids, h].double()[:, None, None])
                    .reshape(-1, D)[:kv] for c in "kv")
            for i in range(h * G, (h + 1) * G):
                w = st["q"][x, i].double() @ K.T * st["scale"]
                if case["causal"]:
                    late = torch.arange(kv, device="cuda")[None, :] > (past + torch.arange(n, device="cuda"))[:, None]
                    w = w.masked_fill(late, -math.inf)
                lse[x, i] = torch.logsumexp(w, -1)
                out[x, i] = torch.exp(w - lse[x, i][:, None]) @ V
    return [out, lse]


def exact(case, seed):
    return (_exact_append if case["op"] == "append" else _exact_attend)(case, seed)
