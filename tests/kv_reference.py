"""Plain 64-bit forms of the decoder cache's two operators, and caches to run them on."""

import math

import torch

LOW, HIGH, TOP = -60, 60, 448.0


def e4m3(y):
    """y (f64) to the nearest e4m3 number, ties to even, saturating; NaN stays."""
    c = y.clamp(-TOP, TOP)
    step = torch.exp2(torch.floor(torch.log2(c.abs().clamp(min=2.0 ** -6))) - 3)
    return torch.round(c / step) * step


def fitting_exponent(amax):
    """The smallest n in [LOW, HIGH] with amax <= 448 * 2^n (python floats)."""
    n = LOW
    while n < HIGH and amax > TOP * 2.0 ** n:
        n += 1
    return n


def rotate(x, cos, sin, rot, interleaved):
    """x [n][H][D], cos and sin [n][rot / 2], in their type: each product and sum rounded to it."""
    x = x.clone()
    f = torch.arange(rot // 2)
    lo, hi = (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)
    a, b = x[..., lo], x[..., hi]
    c, s = cos[:, None], sin[:, None]
    x[..., lo], x[..., hi] = a * c - b * s, b * c + a * s
    return x


class Cache:
    """Numbers of a paged cache in f64 codes and scales, on the host."""

    def __init__(self, pages, heads, P, D, seed=0, stale=None):
        g = torch.Generator().manual_seed(seed)
        self.shape = (pages, heads, P, D)
        self.codes, self.scale = {}, {}
        for n in "kv":
            x = torch.randn(self.shape, generator=g, dtype=torch.float64) * (40 if stale is None else stale)
            self.codes[n] = e4m3(x)
            self.scale[n] = torch.exp2(torch.randint(-8, -3, (pages, heads), generator=g).double())

    def on_gpu(self, wz):
        t = [self.codes[n].float().to(torch.float8_e4m3fn).cuda() for n in "kv"]
        s = [self.scale[n].float().cuda() for n in "kv"]
        return wz.KvCache(*t, *s)

    def clone(self):
        c = Cache.__new__(Cache)
        c.shape = self.shape
        c.codes = {n: x.clone() for n, x in self.codes.items()}
        c.scale = {n: x.clone() for n, x in self.scale.items()}
        return c


def append(cache, k, v, table, cu, start, rotation=None, rot=0, interleaved=False, positions=None, sections=None, q=None,
           work=torch.float64):
    """The operator on the host, in place, rotations in `work`; returns the rotated queries and, for tolerances, the exact
    numbers [(name, page, row, [heads][D])] of the new tokens."""
    P = cache.shape[2]
    q_out = None if q is None else q.to(work).clone()
    exact = []
    for b in range(len(start)):
        x0, x1, s0 = cu[b], cu[b + 1], start[b]
        n = x1 - x0
        if not n:
            continue
        rows = {"k": k[x0:x1].to(work), "v": v[x0:x1].to(work)}
        if rotation is not None:
            half = rot // 2
            tab = rotation.to(work)
            if positions is None:
                pos = torch.arange(s0, s0 + n)[:, None].expand(n, half)
            elif positions.dim() == 1:
                pos = positions[x0:x1].long()[:, None].expand(n, half)
            else:
                pos = torch.repeat_interleave(positions[x0:x1].long(), torch.tensor(sections), 1)
            f = torch.arange(half)
            cos, sin = tab[pos, f], tab[pos, half + f]
            rows["k"] = rotate(rows["k"], cos, sin, rot, interleaved)
            if q is not None:
                q_out[x0:x1] = rotate(q[x0:x1].to(work), cos, sin, rot, interleaved)
        for name, x in rows.items():
            codes, scale = cache.codes[name], cache.scale[name]
            for j in range(s0 // P, (s0 + n - 1) // P + 1):
                page = table[b][j]
                lo, hi = max(s0, j * P), min(s0 + n, (j + 1) * P)
                part = x[lo - s0:hi - s0].transpose(0, 1).double()   # [heads][tokens][D]
                fin = torch.where(torch.isfinite(part), part.abs(), torch.zeros_like(part))
                held = lo - j * P
                for h in range(part.shape[0]):
                    now = 2.0 ** fitting_exponent(fin[h].max().item())
                    old = scale[page, h].item()
                    if held:
                        now = max(now, old)
                        codes[page, h, :held] = e4m3(codes[page, h, :held] * (old / now))
                    codes[page, h, held:hi - j * P] = e4m3(part[h] / now)
                    scale[page, h] = now
                exact.append((name, page, held, part))
    return q_out, exact


def attend(cache, q, table, cu, kv_len, causal, scale):
    """out, lse, and for tolerances sum p |v| / sum p and a bound of the logits' errors, all f64.

    A logit's terms: a query is two e4m3 numbers after a power of two that takes its row's largest
    channel into [128, 256), so a channel is off by at most half the smallest step, 2^-10, of 128;
    sums of D products in fp32 lose at most 2^-20 of their absolute sum."""
    heads, P = cache.shape[1:3]
    T, Hq, D = q.shape
    G = Hq // heads
    out, mass = torch.zeros((2, T, Hq, D), dtype=torch.float64)
    lse = torch.full((T, Hq), -math.inf, dtype=torch.float64)
    off = torch.zeros((T, Hq), dtype=torch.float64)
    for b in range(len(kv_len)):
        x0, n, kv = cu[b], cu[b + 1] - cu[b], kv_len[b]
        if not n or not kv:
            continue
        ids = torch.tensor(table[b][:-(-kv // P)])
        for h in range(heads):
            K, V = ((cache.codes[c][ids, h] * cache.scale[c][ids, h][:, None, None]).reshape(-1, D)[:kv] for c in "kv")
            for i in range(n):
                see = kv - n + i + 1 if causal else kv
                if see <= 0:
                    continue
                qi = q[x0 + i, h * G:(h + 1) * G].double()
                s = qi @ K[:see].T * scale
                top = s.max(-1, keepdim=True).values
                w = torch.exp(s - top)
                total = w.sum(-1, keepdim=True)
                hs = slice(h * G, (h + 1) * G)
                out[x0 + i, hs] = (w / total) @ V[:see]
                mass[x0 + i, hs] = (w / total) @ V[:see].abs()
                lse[x0 + i, hs] = (top + total.log())[:, 0]
                sums = qi.abs() @ K[:see].abs().T * 2.0 ** -20
                step = qi.abs().amax(-1)[:, None] * 2.0 ** -17 * K[:see].abs().sum(-1)[None]
                off[x0 + i, hs] = (sums + step).amax(-1) * abs(scale)
    return out, lse, mass, off
