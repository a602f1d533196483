"""What the operators around the quantized paged cache are timed on: cases, inputs, and each operator in a plain form.

Operators ("op" of a case):
  plan    pages and slots for the new tokens of a batch of requests: a sequence that held `lens` tokens gets `fresh` more;
          the pages that it lacks are taken from the end of a list of free ones, in the order of the sequences
  rotate  queries and keys, per head: n = x w / sqrt(mean x^2 + eps), then the pairs (i, i + rot/2) or (2i, 2i + 1) of its first
          `rot` elements turned by the angle position * frequency_i
  attend  query i of a sequence of L tokens whose last n are new stands at position p = L - n + i and sees the tokens j
          with p - window < j <= p (no window: all up to p): x_j = scale q.k_j, capped to cap * tanh(x_j / cap), plus
          slope_head * (j - p); result sum_j softmax(x)_j v_j and the logarithm of sum_j exp(x_j).  Keys and values lie
          in 8 bits (codes times a step per row of a head) or 4 bits (codes times 2^e per 32 elements) in pages.
"""
import functools
import math

import torch

own = False

BLOCK = 32
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


# ------------------------------------------------------------------------------------------------ cases
def _attend(name, fmt, dtype, seqs, context, new, q_heads, heads, dim, page, window=0, cap=0.0, slopes=False, mixed=False):
    case = {"op": "attend", "format": fmt, "dtype": dtype, "seqs": seqs, "context": context, "new": new, "q_heads": q_heads, "heads": heads,
            "dim": dim, "page": page, "window": window, "cap": cap, "slopes": slopes, "mixed": mixed}
    return {"name": name, **case} if name else case


def listed():
    return [
        # one decoding step of a small batch over short contexts: latency
        _attend("attend_step", "mx4", "bf16", 4, 200, 1, 32, 8, 128, 16),
        # a decoding step of a serving batch, ragged contexts, 8 bits
        _attend("attend_batch", "i8", "bf16", 64, 2000, 1, 32, 8, 128, 64),
        # a decoding step over long contexts, 4 bits: the reading of the cache
        _attend("attend_long", "mx4", "bf16", 8, 32000, 1, 32, 8, 128, 64),
        # one long conversation, one head of keys for eight of queries: one axis to split
        _attend("attend_single", "i8", "f16", 1, 131001, 1, 8, 1, 128, 64),
        # a whole prompt just written: the largest product
        _attend("attend_prompt", "mx4", "bf16", 1, 8192, 8192, 32, 8, 128, 64),
        # chunks of prompts over what went before, capped scores, a sliding window
        _attend("attend_chunk", "i8", "bf16", 4, 16000, 512, 16, 4, 128, 32, window=4096, cap=50.0),
        # chunks of all lengths and single tokens in one batch, odd head size, bias by distance
        _attend("attend_mixed", "mx4", "f16", 24, 3001, 333, 12, 4, 80, 16, slopes=True, mixed=True),
        # one decoding step's projections: latency
        {"name": "rotate_step", "op": "rotate", "tokens": 8, "q_heads": 32, "heads": 8, "dim": 128, "rot": 128, "pairs": False, "norm": True, "far": 30000, "dtype": "bf16"},
        # a prompt's projections
        {"name": "rotate_prompt", "op": "rotate", "tokens": 16384, "q_heads": 32, "heads": 8, "dim": 128, "rot": 128, "pairs": False, "norm": True, "far": 16384, "dtype": "bf16"},
        # part of an odd head turned in neighbouring pairs, 32 bits, far positions
        {"name": "rotate_part", "op": "rotate", "tokens": 1001, "q_heads": 12, "heads": 12, "dim": 80, "rot": 32, "pairs": True, "norm": True, "far": 1000000, "dtype": "f32"},
        # a decoding step's bookkeeping: latency
        {"name": "plan_step", "op": "plan", "seqs": 64, "context": 2000, "new": 1, "page": 64, "spare": 0},
        # many prompts of all lengths, in a buffer of fixed size
        {"name": "plan_prompts", "op": "plan", "seqs": 1500, "context": 1000, "new": 700, "page": 16, "spare": 1777},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the listed ranges: sizes log-uniform and mostly odd, costs below the largest listed case of the operator."""
    op = rng.choice(["attend", "attend", "attend", "rotate", "plan"])
    while op == "attend":
        heads, group, context = rng.choice([1, 2, 3, 4, 8]), rng.choice([1, 2, 4, 5, 8, 16]), _log(rng, 16, 131001)
        case = _attend("", rng.choice(["mx4", "i8"]), rng.choice(["bf16", "bf16", "f16", "f32"]), _log(rng, 1, 64), context,
                       rng.choice([1, 1, _log(rng, 1, 64), _log(rng, 1, min(context, 8192))]), heads * group, heads, rng.choice([64, 80, 96, 128, 128, 256]),
                       rng.choice([16, 32, 64, 128]), window=rng.choice([0, 0, 0, _log(rng, 16, 16384)]), cap=rng.choice([0.0, 0.0, 30.0]),
                       slopes=rng.random() < 0.25, mixed=rng.random() < 0.3)
        if context * case["seqs"] * heads * case["dim"] <= 1 << 27 and case["seqs"] * case["new"] * context * heads * group * case["dim"] <= 1 << 37:
            return case
    if op == "rotate":
        while True:
            dim = rng.choice([64, 80, 96, 128, 256])
            case = {"op": op, "tokens": _log(rng, 1, 16384), "q_heads": rng.choice([1, 4, 8, 12, 32]), "heads": rng.choice([1, 2, 4, 8]), "dim": dim,
                    "rot": rng.choice([dim, dim, dim // 2, 32]), "pairs": rng.random() < 0.5, "norm": rng.random() < 0.75, "far": _log(rng, 1000, 1000000),
                    "dtype": rng.choice(["bf16", "bf16", "f16", "f32"])}
            if case["tokens"] * (case["q_heads"] + case["heads"]) * dim * SIZE[case["dtype"]] <= 168 << 20:
                return case
    while True:
        case = {"op": op, "seqs": _log(rng, 1, 2000), "context": _log(rng, 1, 32000), "new": rng.choice([1, _log(rng, 1, 1000)]), "page": rng.choice([16, 32, 64, 128]),
                "spare": rng.choice([0, _log(rng, 1, 2000)])}
        if case["seqs"] * case["new"] <= 1 << 20 and case["seqs"] * case["context"] // case["page"] <= 1 << 20:
            return case


def _spread(i, most):
    """A number in 0 .. most - 1 that looks arbitrary."""
    return i * 2654435761 % (1 << 32) % most if i else 0


def _lens(case):
    """Tokens in each sequence after the step: the longest has `context`, the others down to half of it."""
    return [case["context"] - _spread(i, case["context"] // 2 + 1) for i in range(case["seqs"])]


def _news(case):
    """New tokens of each sequence: `new`; mixed: every other sequence has one token, the rest any number up to `new`."""
    return [min(c, (1 if i % 2 else case["new"] - _spread(i, case["new"])) if case["mixed"] else case["new"]) for i, c in enumerate(_lens(case))]


def _requests(case):
    """plan: tokens that each sequence held, and that come (some sequences are new, some have nothing to add)."""
    held = [_spread(i + 1, case["context"] + 1) if i % 5 else 0 for i in range(case["seqs"])]
    more = [(0 if i % 7 == 3 else 1) if case["new"] == 1 else _spread(i + 3, case["new"] + 1) for i in range(case["seqs"])]
    return held, more


def _row_bytes(case):
    d = case["dim"]
    return -(-d // BLOCK) * 17 if case["format"] == "mx4" else d + 4


def work(case):
    if case["op"] == "rotate":
        n = case["tokens"] * (case["q_heads"] + case["heads"]) * case["dim"]
        return {"bytes": 2 * n * SIZE[case["dtype"]] + 8 * case["tokens"], "flops": 6 * n}
    if case["op"] == "plan":
        held, more = _requests(case)
        total = sum(more) + case["spare"]
        pages = sum(-(-(h + m) // case["page"]) for h, m in zip(held, more))
        return {"bytes": 16 * total + 40 * case["seqs"] + 8 * pages, "flops": 4 * total}
    w, seen, pairs = case["window"], 0, 0
    for c, n in zip(_lens(case), _news(case)):
        first, last = c - n + 1, c                                   # tokens up to the first and to the last query
        if w:
            seen += min(c, n + w - 1)
            short = max(0, min(last, w) - first + 1)                 # queries that see fewer than w
            pairs += (first + first + short - 1) * short // 2 + (n - short) * w
        else:
            seen += c
            pairs += (first + last) * n // 2
    rows = sum(_news(case))
    return {"bytes": 2 * seen * case["heads"] * _row_bytes(case) + 2 * rows * case["q_heads"] * case["dim"] * SIZE[case["dtype"]] + 4 * rows * case["q_heads"],
            "flops": 4 * pairs * case["q_heads"] * case["dim"]}


# ------------------------------------------------------------------------------------------------ inputs
def _normal(g, *shape):
    return torch.randn(*shape, device="cuda", generator=g)


def _ints(values):
    return torch.tensor(values, device="cuda", dtype=torch.int64)


def _sums(values):
    out = [0]
    for v in values:
        out.append(out[-1] + v)
    return out


def _filled(case, pages, gain, g):
    """Codes and scales of a cache whose rows are normal values, channel d of a head of gain gain[head, d]."""
    page, heads, dim = case["page"], case["heads"], case["dim"]
    codes, scales, step = [], [], max(1, (1 << 26) // (page * heads * dim))
    for p in range(0, pages, step):
        x = _normal(g, min(step, pages - p), page, heads, dim) * gain
        if case["format"] == "mx4":
            e, v = _to_grid(_blocks(x))
            c = (torch.bucketize(v.abs(), torch.tensor(GRID, device="cuda")) + 8 * (v < 0)).to(torch.uint8).flatten(-2)
            codes.append(c[..., 0::2] | (c[..., 1::2] << 4))
            scales.append((e + 127).to(torch.uint8))
        else:
            top = x.abs().amax(-1)
            codes.append((x * (127 / top).unsqueeze(-1)).round().clamp(-127, 127).to(torch.int8))
            scales.append(top / 127)
    return torch.cat(codes), torch.cat(scales)


def _frequencies(rot):
    return (10000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64) / rot)).float().cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    if case["op"] == "rotate":
        n, q, h, d = case["tokens"], case["q_heads"], case["heads"], case["dim"]
        fused = (_normal(g, n, q + 2 * h, d) * torch.exp(0.5 * _normal(g, d))).to(DTYPES[case["dtype"]])       # a projection's output
        state = {"case": case, "q": fused[:, :q], "k": fused[:, q: q + h], "freqs": _frequencies(case["rot"]),
                 "positions": torch.randint(0, case["far"], (n,), device="cuda", generator=g), "q_weight": None, "k_weight": None}
        if case["norm"]:
            state["q_weight"], state["k_weight"] = 1 + 0.2 * _normal(g, d), 1 + 0.2 * _normal(g, d)
        return state
    if case["op"] == "plan":
        held, more = _requests(case)
        page = case["page"]
        have, need = [-(-h // page) for h in held], [-(-(h + m) // page) for h, m in zip(held, more)]
        ids = torch.randperm(sum(need) + 5, device="cuda", generator=g).to(torch.int32)
        width, at = max(need) + 3, sum(have)
        table = torch.full((case["seqs"], width), -1, device="cuda", dtype=torch.int32)
        col = torch.arange(width, device="cuda")
        table[col[None] < _ints(have)[:, None]] = ids[:at]
        return {"case": case, "lens": _ints(held), "fresh": _ints(more), "table": table, "free": ids[at:], "free_count": _ints([ids.numel() - at]),
                "total": sum(more) + case["spare"]}
    heads, dim, page, lens, news = case["heads"], case["dim"], case["page"], _lens(case), _news(case)
    pages = [-(-c // page) for c in lens]
    order = torch.randperm(sum(pages) + 3, device="cuda", generator=g).to(torch.int32)       # a cache that other sequences use too
    table = torch.zeros(len(lens), max(pages), device="cuda", dtype=torch.int32)
    table[torch.arange(max(pages), device="cuda")[None] < _ints(pages)[:, None]] = order[: sum(pages)]
    fused = _normal(g, sum(news), case["q_heads"] + 2 * heads, dim)                           # a projection's output: the queries are a slice of it
    fused *= torch.exp(0.5 * _normal(g, case["q_heads"] + 2 * heads, 1))                      # some heads look closely, some at everything
    state = {"case": case, "q": fused.to(DTYPES[case["dtype"]])[:, : case["q_heads"]], "lens": _ints(lens), "starts": _ints(_sums(news)), "table": table,
             "longest": max(lens), "most": max(news), "slopes": None}                         # the host has made the batch and knows its lengths
    if case["slopes"]:
        state["slopes"] = torch.exp2(-8 * torch.arange(1, case["q_heads"] + 1, device="cuda") / case["q_heads"])
    for n in ("k", "v"):
        gain = torch.exp(0.3 * _normal(g, heads, dim))
        if n == "k":                                                                          # a few channels of keys are far larger
            gain = torch.where(torch.rand(heads, dim, device="cuda", generator=g) < 0.02, 4 * gain, gain)
        state[n + "_codes"], state[n + "_scales"] = _filled(case, order.numel(), gain, g)
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _blocks(x):
    """[..., cols] as [..., blocks, 32], zeros behind the last column."""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))


def _power(e):
    """2^e for whole e in -127..127, exactly."""
    return torch.where(e > -127, (e + 127) << 23, 1 << 22).view(torch.float32)


def _to_grid(x):
    """x [..., 32] in 32 bits -> (exponent of the block's scale [...], elements on the 4-bit grid)."""
    top = x.abs().amax(-1)
    e = torch.where(top > 0, torch.frexp(top).exponent - 3, -127).clamp(-127, 127).to(torch.int32)
    v = x * _power(-e).unsqueeze(-1)
    step = torch.where(v.abs() < 2, 0.5, torch.where(v.abs() < 4, 1.0, 2.0))
    return e, ((v / step).round() * step).clamp(-6, 6)


def _held(s, n, slot):
    """Keys or values of the given slots, in 32 bits [..., heads, dim]."""
    case, codes, scales = s["case"], s[n + "_codes"].flatten(0, 1)[slot], s[n + "_scales"].flatten(0, 1)[slot]
    if case["format"] == "i8":
        return codes.float() * scales.unsqueeze(-1)
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device="cuda")
    v = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (v.unflatten(-1, (-1, BLOCK)) * _power(scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)[..., : case["dim"]]


def _plain_attend(s):
    """Sequences padded to the longest, queries to the most: two batched products around a softmax."""
    case, lens, starts = s["case"], s["lens"], s["starts"]
    seqs, heads, group, dim, page = case["seqs"], case["heads"], case["q_heads"] // case["heads"], case["dim"], case["page"]
    j, i = torch.arange(s["longest"], device="cuda"), torch.arange(s["most"], device="cuda")
    slot = s["table"][:, j // page].long() * page + j % page
    n = starts[1:] - starts[:-1]
    row = (starts[:-1, None] + i).clamp(max=s["q"].shape[0] - 1)                                      # [seqs, most]
    q = s["q"][row].float().unflatten(2, (heads, group)).permute(0, 2, 1, 3, 4).reshape(seqs, heads, -1, dim)
    x = torch.matmul(q, _held(s, "k", slot).permute(0, 2, 3, 1)).mul_(1 / math.sqrt(dim)).unflatten(2, (-1, group))   # [seqs, heads, most, group, longest]
    if case["cap"]:
        x.div_(case["cap"]).tanh_().mul_(case["cap"])
    p = (lens - n)[:, None] + i                                                                       # positions of the queries
    back = j - p.unsqueeze(-1)                                                                        # [seqs, most, longest]
    if case["slopes"]:
        x += s["slopes"].view(1, heads, 1, group, 1) * back[:, None, :, None].float()
    hidden = (back > 0) | (back <= -case["window"]) if case["window"] else back > 0
    x.masked_fill_(hidden[:, None, :, None], -math.inf)
    top = x.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    y = torch.matmul(x.flatten(2, 3), _held(s, "v", slot).transpose(1, 2)).unflatten(2, (-1, group)) / torch.where(total > 0, total, 1.0)
    lse = (total.log() + top).squeeze(-1)
    at = torch.arange(s["q"].shape[0], device="cuda")
    seq = torch.bucketize(at, starts[1:], right=True)
    pick = lambda t: t.transpose(1, 2)[seq, at - starts[seq]].flatten(1, 2)                           # [rows, q_heads, ...]
    return [pick(y).to(s["q"].dtype), pick(lse)]


def _plain_rotate(x, weight, cos, sin, case):
    x, half = x.float(), case["rot"] // 2
    if weight is not None:
        x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * weight
    turn, rest = x[..., : case["rot"]], x[..., case["rot"]:]
    a, b = (turn[..., 0::2], turn[..., 1::2]) if case["pairs"] else (turn[..., :half], turn[..., half:])
    a, b = a * cos - b * sin, b * cos + a * sin
    turn = torch.stack((a, b), -1).flatten(-2) if case["pairs"] else torch.cat((a, b), -1)
    return torch.cat((turn, rest), -1)


def _plain_plan(s):
    case, lens, fresh, total = s["case"], s["lens"], s["fresh"], s["total"]
    page, dev, zero = case["page"], lens.device, lens.new_zeros(1)
    after = lens + fresh
    have, need = (lens + page - 1) // page, (after + page - 1) // page
    first = torch.cat((zero, (need - have).cumsum(0)))                                                # pages that earlier sequences take
    col = torch.arange(s["table"].shape[1], device=dev)
    taken = first[:-1, None] + col - have[:, None]
    count = s["free_count"]
    ids = s["free"][(count - 1 - taken).clamp(0, s["free"].numel() - 1)]
    table = torch.where((col >= have[:, None]) & (col < need[:, None]), torch.where(taken < count, ids, -1), s["table"])
    q_starts, starts = torch.cat((zero, fresh.cumsum(0))), torch.cat((zero, after.cumsum(0)))
    t = torch.arange(total, device=dev)
    seq = torch.bucketize(t, q_starts[1:], right=True)
    inside = seq < lens.numel()
    seq = seq.clamp(max=lens.numel() - 1)
    position = torch.where(inside, lens[seq] + t - q_starts[seq], 0)
    held = table[seq, position // page].long()
    slots = torch.where(inside & (held >= 0), held * page + position % page, -1)
    return [table, after, q_starts, starts, slots, position, (count - first[-1]).clamp(min=0), (first[-1] - count).clamp(min=0)]


def _plain(s):
    case = s["case"]
    if case["op"] == "attend":
        return _plain_attend(s)
    if case["op"] == "plan":
        return _plain_plan(s)
    angle = (s["positions"].double().unsqueeze(-1) * s["freqs"].double()).unsqueeze(1)               # far positions: angles in 64 bits
    cos, sin = angle.cos().float(), angle.sin().float()
    return [_plain_rotate(s["q"], s["q_weight"], cos, sin, case).to(s["q"].dtype), _plain_rotate(s["k"], s["k_weight"], cos, sin, case).to(s["k"].dtype)]


# ------------------------------------------------------------------------------------------------ the framework's calls
@functools.lru_cache(maxsize=None)
def _context():
    import paper_2501_07161_b200 as q

    return q, q.Context(0)


def _own(s):
    q, ctx = _context()
    case = s["case"]
    if case["op"] == "rotate":
        return list(ctx.norm_rotate(s["q"], s["k"], s["positions"], s["freqs"], s["q_weight"], s["k_weight"], eps=EPS, pairs=case["pairs"]))
    if case["op"] == "plan":
        p = ctx.kv_plan(s["lens"], s["fresh"], case["page"], s["table"], s["free"], s["free_count"], s["total"])
        return [s["table"], p.lens, p.q_starts, p.starts, p.slots, p.positions, p.free_count, p.missing]
    if "cache" not in s:
        s["cache"] = q.KvCache({"mx4": q.KV_MX4, "i8": q.KV_I8}[case["format"]], case["dim"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    return list(ctx.kv_attend(s["cache"], s["q"], s["starts"], s["lens"], s["table"], window=case["window"], cap=case["cap"], slopes=s["slopes"],
                              max_new=s["most"], want_lse=True))


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_row(s, n, slot, head):
    """Keys or values [tokens, dim] of one head, by the definition of the format."""
    case = s["case"]
    codes, scales = s[n + "_codes"].flatten(0, 1)[slot, head], s[n + "_scales"].flatten(0, 1)[slot, head]
    if case["format"] == "i8":
        return codes.double() * scales.double().unsqueeze(-1)
    both = torch.stack((codes % 16, codes // 16), -1).reshape(slot.numel(), -1).long()
    grid = torch.tensor(GRID, dtype=torch.float64, device="cuda")
    v = torch.where(both < 8, grid[both % 8], -grid[both % 8])
    return (v * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1))[:, : case["dim"]]


def _exact_attend(s):
    case, group = s["case"], s["case"]["q_heads"] // s["case"]["heads"]
    rows = s["q"].shape[0]
    y = torch.zeros(rows, case["q_heads"], case["dim"], dtype=torch.float64, device="cuda")
    lse = torch.full((rows, case["q_heads"]), -math.inf, dtype=torch.float64, device="cuda")
    at = 0
    for r, (length, new) in enumerate(zip(_lens(case), _news(case))):
        j = torch.arange(length, device="cuda")
        slot = s["table"][r].long()[j // case["page"]] * case["page"] + j % case["page"]
        for h in range(case["heads"]):
            k, v = _exact_row(s, "k", slot, h), _exact_row(s, "v", slot, h)
            step = max(1, (1 << 27) // (length * group))
            for b in range(0, new, step):
                e = min(new, b + step)
                p = torch.arange(length - new + b, length - new + e, device="cuda")
                q = s["q"][at + b: at + e, h * group: (h + 1) * group].double()                        # [queries, group, dim]
                x = (q.reshape(-1, case["dim"]) @ k.T).reshape(e - b, group, length) / math.sqrt(case["dim"])
                if case["cap"]:
                    x = case["cap"] * torch.tanh(x / case["cap"])
                if case["slopes"]:
                    x = x + s["slopes"][h * group: (h + 1) * group].double()[None, :, None] * (j[None] - p[:, None])[:, None].double()
                seen = j[None] <= p[:, None]
                if case["window"]:
                    seen &= j[None] > p[:, None] - case["window"]
                x = torch.where(seen[:, None], x, -math.inf)
                total = torch.logsumexp(x, -1)
                y[at + b: at + e, h * group: (h + 1) * group] = (torch.exp(x - total.unsqueeze(-1)).reshape(-1, length) @ v).reshape(e - b, group, -1)
                lse[at + b: at + e, h * group: (h + 1) * group] = total
        at += new
    return [y, lse]


def _exact_rotate(x, weight, s):
    """Each pair as a complex number times e^(i angle)."""
    case, x = s["case"], x.double()
    if weight is not None:
        x = weight.double() * x * torch.rsqrt((x * x).sum(-1, keepdim=True) / case["dim"] + EPS)
    half = case["rot"] // 2
    i = torch.arange(half, device="cuda")
    first, second = (2 * i, 2 * i + 1) if case["pairs"] else (i, i + half)
    turn = torch.polar(torch.ones(1, dtype=torch.float64, device="cuda"), s["positions"].double()[:, None] * s["freqs"].double())
    z = torch.complex(x[..., first], x[..., second]) * turn[:, None]
    y = x.clone()
    y[..., first], y[..., second] = z.real, z.imag
    return y


def exact(case, seed):
    if case["op"] == "plan":
        return None                                                                                   # whole numbers: they have to be equal
    s = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(s)
    return [_exact_rotate(s["q"], s["q_weight"], s), _exact_rotate(s["k"], s["k_weight"], s)]
