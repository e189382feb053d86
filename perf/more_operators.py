"""Performance cases of a decoder layer's matrix products: what follows the attention over the cache, and what trains
the projector before it.

listed()            the named cases
draw(rng)           one more case of the same ranges
prepare(case, seed) inputs, weights and buffers on the GPU
run(state)          one pass through an operator, and its outputs
work(case)          bytes and flops of one pass that no implementation can do without
exact(case, seed)   the outputs in 64 bits, from torch alone

Four operators on rows of bf16 with weights as torch.nn.Linear has them (out x in) and biases in f32:

  linear           y = act(x W^T + b) + r, with the product before the activation kept where it is asked for
  linear_backward  dx, dW and db of act(x W^T + b) from dy, and from the kept product or from none
  gated            h = act(x Wg^T + bg) * (x Wu^T + bu), with both products kept where they are asked for
  gated_backward   dx, dWg, dWu, dbg and dbu from dh, and from the kept products or from none

`own` chooses the side that run() computes: the plain form (elementary torch operations in 32 bits) or the library's
calls.
"""

import math

import torch

own = False

MOST_ROWS = 18699       # the 18,662 condensed tokens of a 256-frame 27 x 27 video at ratio 0.1, and a question
WIDTH, FEED = 3584, 4 * 3584
ACTS = ("none", "gelu", "gelu_tanh", "silu")


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _linear(name, rows, inner, outer, **kw):
    return {"name": name, "op": "linear", "rows": rows, "in": inner, "out": outer, "act": "none", "bias": False,
            "residual": False, "keep": False, "wide": 0, **kw}


def _linear_backward(name, rows, inner, outer, **kw):
    return {"name": name, "op": "linear_backward", "rows": rows, "in": inner, "out": outer, "act": "none", "bias": True,
            "keep": False, "wide": 0, **kw}


def _gated(name, rows, inner, outer, **kw):
    return {"name": name, "op": "gated", "rows": rows, "in": inner, "out": outer, "act": "silu", "bias": False,
            "keep": False, "wide": 0, **kw}


def _gated_backward(name, rows, inner, outer, **kw):
    return {"name": name, "op": "gated_backward", "rows": rows, "in": inner, "out": outer, "act": "silu", "bias": False,
            "keep": True, "wide": 0, **kw}


def listed():
    return [
        # the attention output of one answer's next token, back into the residual stream: latency
        _linear("linear_token", 1, WIDTH, WIDTH, residual=True),
        # the second product of the feed-forward block for 64 answers' next tokens
        _linear("linear_64_tokens", 64, FEED, WIDTH, residual=True),
        # queries, keys and values (28 + 4 + 4 heads of 128) of a question of 333 tokens
        _linear("linear_question_333", 333, WIDTH, 4608, bias=True),
        # a vision layer's first product in training: seven 27 x 27 frames, odd widths in padded rows
        _linear("linear_frames_odd", 5103, 1151, 4607, act="gelu_tanh", bias=True, keep=True, wide=9),
        # the largest forward product: a video's prompt through the second product of the block
        _linear("linear_prompt_18699", MOST_ROWS, FEED, WIDTH, residual=True),
        # the projector's first layer in training on one long video
        _linear_backward("linear_backward_18662", 18662, WIDTH, WIDTH, act="gelu", keep=True),
        # a linear map of 577 tokens of a smaller encoder: little work on either side of the products
        _linear_backward("linear_backward_577", 577, 1152, WIDTH),
        # the feed-forward block of one answer's next token: both weights read once
        _gated("gated_token", 1, WIDTH, FEED),
        # ... of a question
        _gated("gated_question_333", 333, WIDTH, FEED),
        # ... of a prompt
        _gated("gated_prompt_6151", 6151, WIDTH, FEED),
        # a training step on 4,103 tokens: the largest
        _gated_backward("gated_backward_4103", 4103, WIDTH, FEED),
        # ... of a small block whose products are formed again in the backward pass; ragged widths
        _gated_backward("gated_backward_again_741", 741, 1152, 4616, act="gelu_tanh", bias=True, keep=False, wide=24),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _width(rng):
    kind = rng.random()
    if kind < 0.3:
        return rng.choice([1152, 2304, WIDTH, 4608, FEED])
    n = _log_int(rng, 64, FEED)
    return n // 64 * 64 if kind < 0.55 else n // 8 * 8 if kind < 0.8 else n


def draw(rng):
    make = rng.choice([_linear, _linear, _linear_backward, _gated, _gated_backward])
    case = make("", _log_int(rng, 1, MOST_ROWS), _width(rng), _width(rng))
    case["act"] = rng.choice(ACTS)
    case["bias"] = rng.random() < 0.5
    case["keep"] = rng.random() < 0.5
    case["wide"] = rng.choice([0, 0, 8, 40])
    if "residual" in case:
        case["residual"] = rng.random() < 0.5
    # no dearer than the listed ones
    most = 1.5e12
    row = work({**case, "rows": 1})["flops"]
    case["rows"] = max(1, min(case["rows"], int(most / row)))
    del case["name"]
    return case


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _rows(n, width, wide):
    """An uninitialised [n][width] whose rows begin a multiple of eight elements apart, `wide` or more behind their ends."""
    return torch.empty((n, -(-(width + wide) // 8) * 8), dtype=torch.bfloat16, device="cuda")[:, :width]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    M, K, N, wide = case["rows"], case["in"], case["out"], case["wide"]

    def filled(n, width, gain, pad=wide):
        t = _rows(n, width, pad)
        t.copy_(torch.randn((n, width), generator=g, device="cuda").mul_(gain))
        return t

    # a few channels are strong, as activations have them
    strong = 1 + 4 * (torch.rand(K, generator=g, device="cuda") < 0.02).float()
    s = {"case": case, "x": filled(M, K, strong)}
    both = case["op"].startswith("gated")
    names = ("gate", "up") if both else ("",)
    for name in names:
        s["w" + name] = filled(N, K, 1.3 / math.sqrt(K))
        s["b" + name] = 0.3 * torch.randn(N, generator=g, device="cuda") if case["bias"] else None
    if case["op"].endswith("backward"):
        s["dy"] = filled(M, N, 0.01)
        for name in names:
            s["pre" + name] = filled(M, N, 1.4) if case["keep"] else None
            s["dw" + name] = _rows(N, K, wide)
            s["db" + name] = torch.empty(N, device="cuda") if case["bias"] else None
        s["dx"] = _rows(M, K, wide)
    else:
        s["r"] = filled(M, N, 2.0) if case.get("residual") else None
        s["y"] = _rows(M, N, wide)
        for name in names:
            s["pre" + name] = _rows(M, N, wide) if case["keep"] else None
    return s


# ---------------------------------------------------------------------------
# the plain forms
# ---------------------------------------------------------------------------

_HALF, _TWO_PI = 1 / math.sqrt(2), math.sqrt(2 / math.pi)


def _act(x, act):
    if act == "none":
        return x
    if act == "gelu":
        return 0.5 * x * (1 + torch.erf(x * _HALF))
    if act == "gelu_tanh":
        return 0.5 * x * (1 + torch.tanh(_TWO_PI * (x + 0.044715 * x * x * x)))
    return x / (1 + torch.exp(-x))


def _slope(x, act):
    if act == "gelu":
        return 0.5 * (1 + torch.erf(x * _HALF)) + x * torch.exp(-0.5 * x * x) / math.sqrt(2 * math.pi)
    if act == "gelu_tanh":
        t = torch.tanh(_TWO_PI * (x + 0.044715 * x * x * x))
        return 0.5 * (1 + t) + 0.5 * x * (1 - t * t) * _TWO_PI * (1 + 3 * 0.044715 * x * x)
    s = 1 / (1 + torch.exp(-x))
    return s * (1 + x * (1 - s))


def _product(x, w, b):
    y = torch.matmul(x.float(), w.float().t())
    return y if b is None else y.add_(b)


def _plain(st):
    case, half = st["case"], torch.bfloat16
    op, act = case["op"], case["act"]
    if op == "linear":
        pre = _product(st["x"], st["w"], st["b"])
        y = _act(pre, act)
        if st["r"] is not None:
            y = y + st["r"].float()
        return [y.to(half)] + ([pre.to(half)] if case["keep"] else [])
    if op == "gated":
        g, u = _product(st["x"], st["wgate"], st["bgate"]), _product(st["x"], st["wup"], st["bup"])
        return [(_act(g, act) * u).to(half)] + ([g.to(half), u.to(half)] if case["keep"] else [])
    names = ("gate", "up") if op == "gated_backward" else ("",)
    dy = st["dy"].float()
    if op == "linear_backward" and act == "none":
        d = [dy]
    else:
        pre = [st["pre" + n].float() if case["keep"] else _product(st["x"], st["w" + n], st["b" + n]) for n in names]
        if op == "linear_backward":
            d = [dy * _slope(pre[0], act)]
        else:
            one = torch.ones(())
            d = [dy * pre[1] * (one.to(dy.device) if act == "none" else _slope(pre[0], act)), dy * _act(pre[0], act)]
    x = st["x"].float()
    dx = torch.matmul(d[0], st["w" + names[0]].float())
    if len(d) > 1:
        dx += torch.matmul(d[1], st["w" + names[1]].float())
    out = [dx.to(half)] + [torch.matmul(e.t(), x).to(half) for e in d]
    if case["bias"]:
        out += [e.sum(0, dtype=torch.float64).float() for e in d]
    return out


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _own(st):
    case = st["case"]
    op, act = case["op"], case["act"]
    if "wz" not in st:
        # the binding and the workspace that a program keeps
        import paper_2607_23265_gb300.wavezip as wz
        st["wz"] = wz
        size = {"linear_backward": "wz_linear_backward_workspace_size",
                "gated_backward": "wz_gated_backward_workspace_size"}.get(op)
        if size:
            n = getattr(wz, size)(case["rows"], case["in"], case["out"])
            st["workspace"] = torch.empty(n, dtype=torch.uint8, device="cuda")
    wz = st["wz"]
    if op == "linear":
        y = wz.wz_linear(st["x"], st["w"], st["b"], act=act, residual=st["r"], out=st["y"], pre=st["pre"])
        return [y] + ([st["pre"]] if case["keep"] else [])
    if op == "gated":
        y = wz.wz_gated(st["x"], st["wgate"], st["wup"], st["bgate"], st["bup"], act=act, out=st["y"],
                        gate=st["pregate"], up=st["preup"])
        return [y] + ([st["pregate"], st["preup"]] if case["keep"] else [])
    if op == "linear_backward":
        dx, dw, db = wz.wz_linear_backward(st["dy"], st["x"], st["w"], act=act, bias=st["b"], pre=st["pre"],
                                           need_b=case["bias"], dx=st["dx"], dw=st["dw"], db=st["db"],
                                           workspace=st["workspace"])
        return [dx, dw] + ([db] if case["bias"] else [])
    dx, dwg, dwu, dbg, dbu = wz.wz_gated_backward(
        st["dy"], st["x"], st["wgate"], st["wup"], act=act, b_gate=st["bgate"], b_up=st["bup"], gate=st["pregate"],
        up=st["preup"], need_b=case["bias"], dx=st["dx"], dw_gate=st["dwgate"], dw_up=st["dwup"], db_gate=st["dbgate"],
        db_up=st["dbup"], workspace=st["workspace"])
    return [dx, dwg, dwu] + ([dbg, dbu] if case["bias"] else [])


def run(st):
    return _own(st) if own else _plain(st)


def work(case):
    M, K, N, op = case["rows"], case["in"], case["out"], case["op"]
    both = 2 if op.startswith("gated") else 1
    weights, one = both * N * K * 2, 2 * M * N * K * both
    bias = both * N * 4 if case["bias"] else 0
    if not op.endswith("backward"):
        kept = both if case["keep"] else 0
        rows = 1 + kept + (1 if case.get("residual") else 0)
        return {"bytes": M * K * 2 + weights + bias + rows * M * N * 2, "flops": one + M * N * 10}
    needs = op == "gated_backward" or case["act"] != "none"
    read = both * M * N * 2 if needs and case["keep"] else 0
    again = one if needs and not case["keep"] else 0
    return {"bytes": 2 * M * K * 2 + M * N * 2 + read + 2 * weights + bias * (2 if again else 1),
            "flops": 2 * one + again + M * N * 10 * both}


# ---------------------------------------------------------------------------
# 64 bits
# ---------------------------------------------------------------------------

def _value_and_slope(x, act):
    """The activation and its derivative at x (f64)."""
    if act == "none":
        return x, torch.ones_like(x)
    if act == "silu":
        s = torch.sigmoid(x)
        return x * s, s + x * s * (1 - s)
    if act == "gelu":
        phi = 0.5 * torch.special.erfc(-x / 2 ** 0.5)
        return x * phi, phi + x * torch.exp(-x ** 2 / 2) * (2 * math.pi) ** -0.5
    # 0.5 (1 + tanh z) is the logistic function of 2 z
    z, dz = (2 / math.pi) ** 0.5 * (x + 0.044715 * x ** 3), (2 / math.pi) ** 0.5 * (1 + 0.134145 * x ** 2)
    s = torch.sigmoid(2 * z)
    return x * s, s + x * 2 * s * (1 - s) * dz


def exact(case, seed):
    st = prepare(case, seed)
    op, act = case["op"], case["act"]

    def affine(name):
        y = st["x"].double() @ st["w" + name].double().T
        return y if st["b" + name] is None else y + st["b" + name].double()

    if op == "linear":
        pre = affine("")
        y = _value_and_slope(pre, act)[0]
        if st["r"] is not None:
            y = y + st["r"].double()
        return [y] + ([pre] if case["keep"] else [])
    if op == "gated":
        g, u = affine("gate"), affine("up")
        return [_value_and_slope(g, act)[0] * u] + ([g, u] if case["keep"] else [])
    dy = st["dy"].double()
    if op == "linear_backward":
        if act == "none":
            back = {"": dy}
        else:
            back = {"": dy * _value_and_slope(st["pre"].double() if case["keep"] else affine(""), act)[1]}
    else:
        g, u = (st["pre" + n].double() if case["keep"] else affine(n) for n in ("gate", "up"))
        a, da = _value_and_slope(g, act)
        back = {"gate": dy * u * da, "up": dy * a}
    dx = sum(d @ st["w" + n].double() for n, d in back.items())
    return [dx] + [d.T @ st["x"].double() for d in back.values()] + ([d.sum(0) for d in back.values()] if case["bias"] else [])
