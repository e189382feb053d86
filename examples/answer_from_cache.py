"""Condense a video, put its tokens in a decoder's 8-bit cache, attend to them, and run a layer.

What a serving program does around one layer of an LLM: the condensed and projected tokens take
positions from the index map (frame, row, column), the question's tokens follow with all three axes
alike, one product gives queries, keys and values, the prompt attends to itself causally, the
attention's output goes back into the residual stream and through a gated feed-forward block,
and then single tokens are appended and answered one by one.  Weights and inputs are random: the program
shows the calls and checks them against plain attention and plain products in fp32.

    python examples/answer_from_cache.py
"""

import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2607_23265_gb300.wavezip as wz  # noqa: E402


def plain_attention(q, cache, pages, kv_len, causal):
    """[n, Hq, D] attention over the first kv_len slots of the cache's numbers, in fp32."""
    D, heads = cache.D, cache.heads
    used = pages[:-(-kv_len // cache.page_tokens)].long()
    k, v = ((c.float()[used] * s[used][:, :, None, None]).permute(1, 0, 2, 3).reshape(heads, -1, D)[:, :kv_len]
            for c, s in ((cache.k, cache.k_scale), (cache.v, cache.v_scale)))
    n, Hq, _ = q.shape
    w = torch.einsum("nhgd,htd->hgnt", q.float().view(n, heads, Hq // heads, D), k) / math.sqrt(D)
    if causal:
        late = torch.arange(kv_len, device=q.device)[None] > (kv_len - n + torch.arange(n, device=q.device))[:, None]
        w = w.masked_fill(late, -math.inf)
    return torch.einsum("hgnt,htd->nhgd", w.softmax(-1), v).reshape(n, Hq, D)


def plain_layer(rows, o, w_o, w_gate, w_up, w_down):
    """What follows the attention's output o of a layer's rows, in fp32."""
    x = rows.float() + o.float() @ w_o.float().T
    g = x @ w_gate.float().T
    return x + (g * torch.sigmoid(g) * (x @ w_up.float().T)) @ w_down.float().T


def main(T=16, H=13, W=13, D=512, Hq=8, heads=2, head_dim=64, page=64, question=21, answer=5, seed=0):
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    rand = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731

    # the video's tokens, and where they come from
    video, query = rand(T, H, W, D).bfloat16(), (rand(question, D) / math.sqrt(D)).bfloat16()
    out = wz.wz_condense_ex(video, query, 0.25)
    n = int(out["count"])
    w1, w2 = ((rand(D, D) / math.sqrt(D)).bfloat16() for _ in range(2))
    tokens = wz.wz_project(out["tokens"][:n], w1, None, w2, None)

    # the prompt: condensed tokens at (t, i, j), then the question
    prompt = torch.cat([tokens, query])
    last = T + torch.arange(question, device=dev, dtype=torch.int32)
    positions = torch.cat([out["index"][:n], last[:, None].expand(-1, 3)]).contiguous()
    wide = Hq * head_dim
    weight = lambda outs, ins: (rand(outs, ins) / math.sqrt(ins)).bfloat16()  # noqa: E731
    w_qkv, b_qkv = weight(wide + 2 * heads * head_dim, D), 0.1 * rand(wide + 2 * heads * head_dim)
    w_o, w_gate, w_up, w_down = weight(D, wide), weight(4 * D, D), weight(4 * D, D), weight(D, 4 * D)

    # a cache with room for the answer; this sequence's pages lie anywhere in it
    length = prompt.shape[0]
    need = -(-(length + answer) // page)
    cache = wz.KvCache.empty(need + 3, heads, page, head_dim)
    table = torch.randperm(need + 3, generator=g, device=dev)[:need].to(torch.int32)[None]
    rotation = wz.rotation_table(T + question + answer, head_dim)
    sections = [8, 12, 12]                                   # frequencies for t, i and j
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device=dev)  # noqa: E731
    status = torch.zeros(1, dtype=torch.int32, device=dev)
    workspace = torch.empty(wz.wz_attend_workspace_size(length, Hq, head_dim), dtype=torch.uint8, device=dev)

    worst = 0.0
    held = 0
    rows = prompt
    for step in range(1 + answer):
        new = rows.shape[0]
        qkv = wz.wz_linear(rows, w_qkv, b_qkv).view(new, Hq + 2 * heads, head_dim)
        q = wz.wz_kv_append(qkv[:, Hq:Hq + heads], qkv[:, Hq + heads:], cache, table, i32(0, new), i32(held), max_new=new,
                            q=qkv[:, :Hq], rotation=rotation, positions=positions, sections=sections,
                            device_status=status)
        held += new
        o = wz.wz_attend(q, cache, table, i32(0, new), i32(held), max_new=new, workspace=workspace, device_status=status)
        want = plain_attention(q, cache, table[0], held, True)
        worst = max(worst, float((o.float() - want).norm() / want.norm()))
        o = o.view(new, wide)
        x = wz.wz_linear(o, w_o, residual=rows)
        y = wz.wz_linear(wz.wz_gated(x, w_gate, w_up), w_down, residual=x)
        want = plain_layer(rows, o, w_o, w_gate, w_up, w_down)
        worst = max(worst, float((y.float() - want).norm() / want.norm()))
        rows = y[-1:] / y[-1:].float().std().bfloat16()                                     # the next token's input
        positions = (last[-1] + 1 + i32(step))[:, None].expand(1, 3).contiguous()
    assert int(status) == 0, f"status {int(status):#x}"
    print(f"{n} condensed tokens and {question} of the question cached, {answer} tokens answered: "
          f"outputs within {worst:.1e} of plain attention and products")
    return worst


if __name__ == "__main__":
    main()
