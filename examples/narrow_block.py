"""A transformer block run in 4 bits: how far each of its outputs is from FP32, and which layers to leave there.

A block of random weights (attention over a quantized paged cache, then a layer of experts) decodes a few tokens after a
prompt, once in FP32 with plain torch operations and once through the 4-bit layers and the cache.  The framework's own
metrics then compare every stage's output, and its ranking says which layers lose most.

    python examples/narrow_block.py [--cache mx4|i8]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_07161_b200 as q  # noqa: E402

WIDTH, HEADS, KV_HEADS, DIM, EXPERTS, TOP, INNER, PAGE = 512, 8, 2, 64, 8, 2, 768, 16


def attention(x, k, v, lens):
    """x [tokens, HEADS * DIM] queries, one per token in order; k, v whole sequences one after the other; lens: tokens of each
    sequence, its last `new` ones being the queries."""
    out, at, row = torch.empty_like(x), 0, 0
    for total, new in lens:
        qs = x[row: row + new].view(new, KV_HEADS, HEADS // KV_HEADS, DIM)
        ks, vs = k[at: at + total], v[at: at + total]
        s = torch.einsum("thgd,shd->thgs", qs, ks) / DIM ** 0.5
        late = torch.arange(total, device=x.device)[None] > torch.arange(total - new, total, device=x.device)[:, None]
        s = s.masked_fill(late[:, None, None], float("-inf")).softmax(-1)
        out[row: row + new] = torch.einsum("thgs,shd->thgd", s, vs).reshape(new, HEADS * DIM)
        at, row = at + total, row + new
    return out


class Block:
    """The same weights in FP32 and in 4 bits."""

    def __init__(self, ctx, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        make = lambda *s: torch.randn(*s, device="cuda", generator=g) / s[-1] ** 0.5
        self.ctx = ctx
        self.w = {"qkv": make((HEADS + 2 * KV_HEADS) * DIM, WIDTH), "out": make(WIDTH, HEADS * DIM),
                  "up": make(EXPERTS, INNER, WIDTH), "down": make(EXPERTS, WIDTH, INNER)}
        self.router = make(EXPERTS, WIDTH)
        self.narrow = {}
        for name, w in self.w.items():
            m = ctx.mx_quantize(w)                                     # rows of all experts one after the other
            if w.dim() == 3:                                           # ... then one matrix per expert
                m = q.MxMatrix(m.codes.view(*w.shape[:2], -1), m.scales.unflatten(0, w.shape[:2]), m.cols)
            self.narrow[name] = m

    def experts(self, x, linear):
        """Tokens to their TOP experts: rows sorted by expert, two grouped products, rows added up again."""
        weight, expert = (x.float() @ self.router.T).softmax(-1).topk(TOP, -1)
        order = expert.flatten().argsort(stable=True)
        offsets = torch.nn.functional.pad(torch.bincount(expert.flatten(), minlength=EXPERTS).cumsum(0), (1, 0))
        rows = x[order // TOP]
        up = linear("up", rows, offsets)
        down = linear("down", torch.nn.functional.silu(up), offsets)
        return up, torch.zeros_like(x).index_add_(0, order // TOP, down * weight.flatten()[order, None].to(down.dtype)), (order, offsets)


def run(ctx, cache_format=q.KV_MX4, prompts=(70, 33, 1, 128), steps=3, seed=0):
    """-> {stage: (FP32 output, 4-bit output)} of the last step, and the block."""
    block = Block(ctx, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    pages = [-(-(p + steps) // PAGE) for p in prompts]
    ids = torch.randperm(sum(pages), device="cuda", generator=g).to(torch.int32)
    table = torch.zeros(len(prompts), max(pages), dtype=torch.int32, device="cuda")
    for i, n in enumerate(pages):
        table[i, :n] = ids[sum(pages[:i]): sum(pages[: i + 1])]
    cache = ctx.kv_empty(sum(pages), PAGE, KV_HEADS, DIM, cache_format)
    past = [torch.empty(0, 2 * KV_HEADS, DIM, device="cuda") for _ in prompts]          # FP32 keys and values
    lens = [0] * len(prompts)
    for step in range(steps + 1):
        new = list(prompts) if step == 0 else [1] * len(prompts)
        x = torch.randn(sum(new), WIDTH, device="cuda", generator=g)
        slots = torch.cat([table[i, torch.arange(n, n + c, device="cuda") // PAGE].long() * PAGE + torch.arange(n, n + c, device="cuda") % PAGE
                           for i, (n, c) in enumerate(zip(lens, new))])
        lens = [n + c for n, c in zip(lens, new)]
        starts = torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device="cuda")
        both = list(zip(lens, new))

        qkv = x @ block.w["qkv"].T
        kv = qkv[:, HEADS * DIM:].view(-1, 2 * KV_HEADS, DIM)
        past = [torch.cat((p, part)) for p, part in zip(past, kv.split(new))]
        every = torch.cat(past)
        att = attention(qkv[:, : HEADS * DIM], every[:, :KV_HEADS], every[:, KV_HEADS:], both)
        out = att @ block.w["out"].T

        def plain(name, rows, offsets):
            o = offsets.tolist()
            return torch.cat([rows[o[e]: o[e + 1]] @ block.w[name][e].T for e in range(EXPERTS)])
        up, moe, (order, offsets) = block.experts(x + out, plain)

        h = x.bfloat16()
        nqkv = ctx.mx_linear(h, block.narrow["qkv"])
        nkv = nqkv[:, HEADS * DIM:].unflatten(1, (2 * KV_HEADS, DIM))
        ctx.kv_write(cache, nkv[:, :KV_HEADS], nkv[:, KV_HEADS:], slots)
        k, v = ctx.kv_read(cache, table, starts, sum(lens))
        natt = attention(nqkv[:, : HEADS * DIM].float(), k.float(), v.float(), both)
        nout = ctx.mx_linear(natt.bfloat16(), block.narrow["out"])
        # the experts of the FP32 pass, so that a token that changes sides does not drown the layers' own error
        rows = (h + nout)[order // TOP]
        nup = ctx.mx_linear_grouped(rows, offsets, block.narrow["up"])
        weight = ((x + out) @ block.router.T).softmax(-1).topk(TOP, -1)[0].flatten()[order, None]
        ndown = ctx.mx_linear_grouped(torch.nn.functional.silu(nup), offsets, block.narrow["down"])
        nmoe = torch.zeros_like(x).index_add_(0, order // TOP, ndown.float() * weight)
    return {"qkv": (qkv, nqkv.float()), "out": (out, nout.float()), "up": (up, nup.float()), "down": (moe, nmoe)}, block


def report(ctx, stages, block):
    """SQNR of each layer's weights and of its output, and the layers in order of sensitivity."""
    descs, keep = [], []
    for name, w in block.w.items():                                    # weights against their 4-bit copies
        pair = (w.reshape(-1, w.shape[-1]), ctx.mx_dequantize(block.narrow[name]).reshape(-1, w.shape[-1]))
        keep.append(pair)
    keep += [tuple(t.contiguous() for t in pair) for pair in stages.values()]
    for a, b in keep:
        descs.append(q.make_desc(a, b, 1, *a.shape, q.PER_TENSOR, q.SYM_I8, flags=q.PAIR_RAW))
    descs = q.desc_array(descs)
    cal = ctx.calibrate(descs, want_hist=False)
    met = ctx.quant_metrics(descs, cal.step, cal.inv, cal.offset)
    n = len(stages)
    order, _, _ = ctx.rank_layers(met.sqnr_db[:n].contiguous(), met.mse[:n].contiguous(), met.sqnr_db[n:].contiguous(), met.mse[n:].contiguous())
    return met.sqnr_db[:n].tolist(), met.sqnr_db[n:].tolist(), order.tolist()


def main():
    ap = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    ap.add_argument("--cache", choices=("mx4", "i8"), default="mx4")
    a = ap.parse_args()
    ctx = q.Context(0)
    stages, block = run(ctx, q.KV_MX4 if a.cache == "mx4" else q.KV_I8)
    w, x, order = report(ctx, stages, block)
    for i, name in enumerate(stages):
        print("%-5s weights %5.1f dB  output %5.1f dB" % (name, w[i], x[i]))
    print("most sensitive first:", ", ".join(list(stages)[i] for i in order))
    ctx.close()


if __name__ == "__main__":
    main()
