"""What the microscaled 4-bit operators and the quantized cache are timed on: cases, inputs, and each operator in a plain form.

The 4-bit format holds a row in blocks of 32 elements.  With A the largest magnitude of a block, the block's scale is
2^e, e = floor(log2 A) - 2, stored as the byte e + 127, and each element is x * 2^-e rounded to the nearest of
0, 0.5, 1, 1.5, 2, 3, 4, 6 (ties to the even code, magnitudes over 6 become 6), stored as a 4-bit code with the sign on
top.  The 8-bit cache holds a row of one head as round(x * 127 / R) with R the row's largest magnitude, and R / 127.

Operators ("op" of a case):
  quantize  x [rows, cols] to 4 bits, returned as the values that the codes stand for
  linear    y = q(x) w^T + bias with w held in 4 bits
  grouped   the same where consecutive runs of rows belong to experts, each with a weight of its own
  cache     keys and values of new tokens written to a paged cache, and whole sequences read back from it
"""
import functools
import math

import torch

own = False

BLOCK = 32
DTYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one token's hidden state, as every decoding step quantizes it
        {"name": "quantize_token", "op": "quantize", "rows": 1, "cols": 4096, "dtype": "bf16"},
        # activations of a prompt before a projection
        {"name": "quantize_prompt", "op": "quantize", "rows": 16384, "cols": 8192, "dtype": "bf16"},
        # a calibration batch of VGG-16's fc6 inputs, stored in 32 bits, rows that end inside a vector load's stride
        {"name": "quantize_fc6_f32", "op": "quantize", "rows": 1001, "cols": 25088, "dtype": "f32"},
        # one image through VGG-16's fc6: the call is the reading of 53 MB of weights
        {"name": "linear_fc6_single", "op": "linear", "rows": 1, "cols": 25088, "out": 4096, "dtype": "bf16", "bias": True},
        # a decoding batch through a square projection
        {"name": "linear_decode_64", "op": "linear", "rows": 64, "cols": 4096, "out": 4096, "dtype": "bf16", "bias": False},
        # VGG-16's fc8 for a ragged batch: 1000 outputs, half precision
        {"name": "linear_fc8_ragged", "op": "linear", "rows": 333, "cols": 4096, "out": 1000, "dtype": "f16", "bias": True},
        # a long prompt through a large projection: the largest product
        {"name": "linear_prompt", "op": "linear", "rows": 8192, "cols": 8192, "out": 8192, "dtype": "bf16", "bias": False},
        # 16 tokens, four experts each, at a decoding step: a few rows per expert, some experts without any
        {"name": "grouped_decode", "op": "grouped", "rows": 64, "cols": 2048, "out": 4096, "experts": 32, "dtype": "bf16", "bias": False},
        # a prompt's tokens sorted by expert, ragged runs
        {"name": "grouped_prompt", "op": "grouped", "rows": 16411, "cols": 2048, "out": 4096, "experts": 16, "dtype": "bf16", "bias": True},
        # one decoding step of a small batch: a token written per sequence, short contexts read back, 4 bits
        {"name": "cache_step", "op": "cache", "seqs": 4, "context": 200, "new": 1, "heads": 8, "dim": 128, "page": 16, "format": "mx4", "dtype": "bf16"},
        # prompts of 32 sequences written and read back in 8 bits
        {"name": "cache_prompt", "op": "cache", "seqs": 32, "context": 1000, "new": 1000, "heads": 8, "dim": 128, "page": 64, "format": "i8", "dtype": "bf16"},
        # long contexts read back at a decoding step, 4 bits
        {"name": "cache_long", "op": "cache", "seqs": 8, "context": 32000, "new": 1, "heads": 8, "dim": 128, "page": 64, "format": "mx4", "dtype": "bf16"},
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the listed ranges: sizes log-uniform and mostly odd, costs below the largest listed case of the operator."""
    op = rng.choice(["quantize", "linear", "linear", "grouped", "cache"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    while True:
        if op == "quantize":
            case = {"op": op, "rows": _log(rng, 1, 16384), "cols": _log(rng, 64, 25088), "dtype": dtype}
            if case["rows"] * case["cols"] <= 1 << 26:
                return case
        elif op == "linear":
            case = {"op": op, "rows": _log(rng, 1, 8192), "cols": _log(rng, 256, 25088), "out": _log(rng, 256, 8192),
                    "dtype": rng.choice(["bf16", "f16"]), "bias": rng.random() < 0.5}
            if case["rows"] * case["cols"] * case["out"] <= 1 << 38 and case["cols"] * case["out"] <= 1 << 27:
                return case
        elif op == "grouped":
            case = {"op": op, "rows": _log(rng, 8, 16411), "cols": _log(rng, 256, 4096), "out": _log(rng, 256, 4096),
                    "experts": _log(rng, 2, 64), "dtype": rng.choice(["bf16", "f16"]), "bias": rng.random() < 0.5}
            if case["rows"] * case["cols"] * case["out"] <= 1 << 36 and case["cols"] * case["out"] * case["experts"] <= 1 << 28:
                return case
        else:
            context = _log(rng, 16, 32000)
            case = {"op": op, "seqs": _log(rng, 1, 64), "context": context, "new": rng.choice([1, 1, context, _log(rng, 1, context)]),
                    "heads": rng.choice([1, 2, 4, 8, 16]), "dim": rng.choice([64, 80, 96, 128, 256]), "page": rng.choice([16, 32, 64, 128]),
                    "format": rng.choice(["mx4", "i8"]), "dtype": rng.choice(["bf16", "f16"])}
            if case["seqs"] * context * case["heads"] * case["dim"] <= 8 * 32000 * 8 * 128:
                return case


def _counts(case):
    """Rows per expert: shares that fall off with a power law, dealt in a fixed odd order; with few rows some get none."""
    e, rows = case["experts"], case["rows"]
    order = sorted(range(e), key=lambda i: (i * 7919 + 13) % 104729)
    share = [1.0 / math.sqrt(1 + order[i]) for i in range(e)]
    total, got, acc, out = sum(share), 0, 0.0, []
    for i in range(e):
        acc += share[i]
        upto = rows if i == e - 1 else int(rows * acc / total)
        out.append(upto - got)
        got = upto
    return out


def _contexts(case):
    """Tokens in each sequence after the step: the longest has `context`, the others down to half of it."""
    n, c = case["seqs"], case["context"]
    return [max(1, c - (i * 2654435761 % (c // 2 + 1) if i else 0)) for i in range(n)]


def _row_bytes(case):
    d = case["dim"]
    blocks = -(-d // BLOCK)
    return blocks * 17 if case["format"] == "mx4" else d + 4


def work(case):
    if case["op"] == "quantize":
        n = case["rows"] * case["cols"]
        return {"bytes": n * (2 * SIZE[case["dtype"]] + 0.5 + 1 / BLOCK), "flops": 2 * n}
    if case["op"] in ("linear", "grouped"):
        m, k, n, s = case["rows"], case["cols"], case["out"], SIZE[case["dtype"]]
        used = sum(c > 0 for c in _counts(case)) if case["op"] == "grouped" else 1
        bias = 4 * n * used if case["bias"] else 0
        return {"bytes": m * k * s + used * n * k * (0.5 + 1 / BLOCK) + m * n * s + bias, "flops": 2 * m * n * k}
    lens = _contexts(case)
    new, total = sum(min(case["new"], c) for c in lens), sum(lens)
    rows, wide = case["heads"] * 2, case["dim"] * SIZE[case["dtype"]]
    return {"bytes": rows * (new * (wide + _row_bytes(case)) + total * (wide + _row_bytes(case))), "flops": 2 * rows * case["dim"] * (new + total)}


# ------------------------------------------------------------------------------------------------ inputs
def _rng(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    return g


def _activations(rows, cols, dtype, g):
    """Normal values with a few channels an order of magnitude larger, as hidden states have them."""
    gain = torch.exp(0.3 * torch.randn(cols, device="cuda", generator=g))
    gain = torch.where(torch.rand(cols, device="cuda", generator=g) < 0.01, 12 * gain, gain)
    return (torch.randn(rows, cols, device="cuda", generator=g) * gain).to(DTYPES[dtype])


def _weights(shape, g):
    """Codes and scales of normal weights of standard deviation 1 / sqrt(cols); scale rows padded to 16 bytes, as a checkpoint's loader lays them out."""
    cols = shape[-1]
    blocks = -(-cols // BLOCK)
    w = torch.randn(*shape, device="cuda", generator=g) / math.sqrt(cols)
    scale, q = _to_grid(_blocks(w))
    code = torch.bucketize(q.abs(), torch.tensor(GRID, device="cuda")).to(torch.uint8) + 8 * (q < 0).to(torch.uint8)
    code = code.flatten(-2)
    codes = (code[..., 0::2] | (code[..., 1::2] << 4)).contiguous()
    scales = torch.zeros(*shape[:-1], -(-blocks // 16) * 16, device="cuda", dtype=torch.uint8)
    scales[..., :blocks] = (scale + 127).to(torch.uint8)
    return codes, scales[..., :blocks]


def prepare(case, seed):
    g = _rng(case, seed)
    if case["op"] == "quantize":
        return {"case": case, "x": _activations(case["rows"], case["cols"], case["dtype"], g)}
    if case["op"] in ("linear", "grouped"):
        experts = (case["experts"],) if case["op"] == "grouped" else ()
        state = {"case": case, "x": _activations(case["rows"], case["cols"], case["dtype"], g), "bias": None}
        state["codes"], state["scales"] = _weights((*experts, case["out"], case["cols"]), g)
        if case["bias"]:
            state["bias"] = torch.randn(*experts, case["out"], device="cuda", generator=g)
        if experts:
            counts = _counts(case)
            state["offsets"] = torch.tensor([sum(counts[:i]) for i in range(len(counts) + 1)], device="cuda")
            state["most"] = max(counts)  # the host knows the run lengths: it has sorted the tokens
        return state
    heads, dim, page, lens = case["heads"], case["dim"], case["page"], _contexts(case)
    pages = [-(-c // page) for c in lens]
    order = torch.randperm(sum(pages) + 3, device="cuda", generator=g)  # a cache that other sequences use too
    table = torch.zeros(len(lens), max(pages), device="cuda", dtype=torch.int32)
    slots = []
    for i, c in enumerate(lens):
        mine = order[sum(pages[:i]): sum(pages[: i + 1])]
        table[i, : pages[i]] = mine.to(torch.int32)
        at = torch.arange(c - min(case["new"], c), c, device="cuda")
        slots.append(mine[at // page] * page + at % page)
    slots = torch.cat(slots)
    fused = torch.randn(slots.numel(), 3 * heads, dim, device="cuda", generator=g).to(DTYPES[case["dtype"]])  # a projection's output: keys and values are slices of it
    shape = (order.numel(), page, heads)
    state = {"case": case, "k": fused[:, heads: 2 * heads], "v": fused[:, 2 * heads:], "slots": slots, "table": table, "total": sum(lens),
             "starts": torch.tensor([sum(lens[:i]) for i in range(len(lens) + 1)], device="cuda")}
    blocks = -(-dim // BLOCK)
    for n in ("k", "v"):  # what earlier steps have written
        if case["format"] == "mx4":
            state[n + "_codes"] = torch.randint(0, 256, (*shape, blocks * BLOCK // 2), device="cuda", generator=g, dtype=torch.uint8)
            state[n + "_scales"] = torch.randint(124, 127, (*shape, blocks), device="cuda", generator=g, dtype=torch.uint8)
        else:
            state[n + "_codes"] = torch.randint(-127, 128, (*shape, dim), device="cuda", generator=g, dtype=torch.int8)
            state[n + "_scales"] = 0.02 + 0.01 * torch.rand(*shape, device="cuda", generator=g)
    return state


# ------------------------------------------------------------------------------------------------ plain forms
def _blocks(x):
    """[..., cols] as [..., blocks, 32], zeros behind the last column."""
    short = -x.shape[-1] % BLOCK
    return torch.nn.functional.pad(x, (0, short)).unflatten(-1, (-1, BLOCK))


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


def _round_trip(x):
    """The values of x [..., cols] after its rounding to 4 bits, in 32 bits."""
    e, q = _to_grid(_blocks(x.float()))
    return (q * _power(e).unsqueeze(-1)).flatten(-2)[..., : x.shape[-1]]


def _values(codes, scales, cols):
    """The values that packed codes and scale bytes stand for, in 32 bits."""
    grid = torch.tensor(GRID + tuple(-v for v in GRID), device=codes.device)
    q = grid[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()]
    return (q.unflatten(-1, (-1, BLOCK)) * _power(scales.to(torch.int32) - 127).unsqueeze(-1)).flatten(-2)[..., :cols]


def _plain(s):
    case = s["case"]
    if case["op"] == "quantize":
        return _round_trip(s["x"]).to(s["x"].dtype)
    if case["op"] == "linear":
        y = _round_trip(s["x"]) @ _values(s["codes"], s["scales"], case["cols"]).T
        return (y if s["bias"] is None else y + s["bias"]).to(s["x"].dtype)
    if case["op"] == "grouped":  # every run padded to the longest, one batched product, the rows picked out again
        row = torch.arange(case["rows"], device="cuda")
        expert = torch.bucketize(row, s["offsets"][1:], right=True)
        place = row - s["offsets"][expert]
        padded = torch.zeros(case["experts"], s["most"], case["cols"], device="cuda")
        padded[expert, place] = _round_trip(s["x"])
        y = torch.bmm(padded, _values(s["codes"], s["scales"], case["cols"]).transpose(1, 2))[expert, place]
        return (y if s["bias"] is None else y + s["bias"][expert]).to(s["x"].dtype)
    heads, dim, page = case["heads"], case["dim"], case["page"]
    row = torch.arange(s["total"], device="cuda")
    seq = torch.bucketize(row, s["starts"][1:], right=True)
    at = row - s["starts"][seq]
    place = s["table"][seq, at // page].long() * page + at % page
    out = []
    for n in ("k", "v"):  # keys and values go through the same steps
        x, codes, scales = s[n].float(), s[n + "_codes"].flatten(0, 1), s[n + "_scales"].flatten(0, 1)
        if case["format"] == "mx4":
            e, q = _to_grid(_blocks(x))
            code = (torch.bucketize(q.abs(), torch.tensor(GRID, device="cuda")) + 8 * (q < 0)).to(torch.uint8).flatten(-2)
            codes[s["slots"]] = code[..., 0::2] | (code[..., 1::2] << 4)
            scales[s["slots"]] = (e + 127).to(torch.uint8)
            y = _values(codes[place], scales[place], dim)
        else:
            top = x.abs().amax(-1)
            inv = torch.where(top > 0, 127 / top, 0.0)
            codes[s["slots"]] = (x * inv.unsqueeze(-1)).round().clamp(-127, 127).to(torch.int8)
            scales[s["slots"]] = top / 127
            y = codes[place].float() * scales[place].unsqueeze(-1)
        out.append(y.to(s[n].dtype))
    return out


# ------------------------------------------------------------------------------------------------ the framework's calls
@functools.lru_cache(maxsize=None)
def _context():
    import paper_2501_07161_b200 as q

    return q, q.Context(0)


def _own(s):
    q, ctx = _context()
    case = s["case"]
    if case["op"] == "quantize":
        return ctx.mx_quantize(s["x"], want_values=True).values
    if case["op"] in ("linear", "grouped"):
        if "weight" not in s:
            s["weight"] = q.MxMatrix(s["codes"], s["scales"], case["cols"])
        if case["op"] == "linear":
            return ctx.mx_linear(s["x"], s["weight"], bias=s["bias"])
        return ctx.mx_linear_grouped(s["x"], s["offsets"], s["weight"], bias=s["bias"])
    if "cache" not in s:
        s["cache"] = q.KvCache({"mx4": q.KV_MX4, "i8": q.KV_I8}[case["format"]], case["dim"], s["k_codes"], s["k_scales"], s["v_codes"], s["v_scales"])
    ctx.kv_write(s["cache"], s["k"], s["v"], s["slots"])
    return list(ctx.kv_read(s["cache"], s["table"], s["starts"], s["total"], s["k"].dtype))


def run(state):
    return _own(state) if own else _plain(state)


# ------------------------------------------------------------------------------------------------ in 64 bits
def _exact_round_trip(x):
    """By the definition: the nearest grid point (the even code of two that are equally near), in 64 bits."""
    rows, cols = x.reshape(-1, x.shape[-1]).shape
    out = torch.empty(rows, cols, dtype=torch.float64, device=x.device)
    grid = torch.tensor(GRID, dtype=torch.float64, device=x.device)
    middle = (grid[1:] + grid[:-1]) / 2
    for r in range(0, rows, 2048):
        part = x.reshape(-1, cols)[r: r + 2048].double()
        for c in range(0, cols, 8192):
            b = _blocks(part[:, c: c + 8192])
            top = b.abs().amax(-1, keepdim=True)
            mantissa, exponent = torch.frexp(top)  # top = mantissa * 2^exponent, 1/2 <= mantissa < 1; log2 in 64 bits misses whole powers
            scale = torch.where(top > 0, top / torch.where(top > 0, mantissa, 1.0) / 8, 1.0)
            v = b.abs() / scale
            below, above = torch.bucketize(v, middle), torch.bucketize(v, middle, right=True)
            code = torch.where(below % 2 == 0, below, above)  # they differ only at a tie
            out[r: r + 2048, c: c + 8192] = (torch.sign(b) * grid[code] * scale).flatten(-2)[:, : min(8192, cols - c)]
    return out.reshape(x.shape)


def _exact_values(codes, scales, cols):
    low, high = (codes % 16).long(), (codes // 16).long()
    both = torch.stack((low, high), -1).reshape(*codes.shape[:-1], -1)
    grid = torch.tensor(GRID, dtype=torch.float64, device=codes.device)
    q = torch.where(both < 8, grid[both % 8], -grid[both % 8])[..., :cols]
    return q * torch.exp2(scales.double() - 127).repeat_interleave(BLOCK, -1)[..., :cols]


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "quantize":
        return _exact_round_trip(s["x"])
    if case["op"] == "linear":
        y = _exact_round_trip(s["x"]) @ _exact_values(s["codes"], s["scales"], case["cols"]).T
        return y if s["bias"] is None else y + s["bias"].double()
    if case["op"] == "grouped":
        x, at, parts = _exact_round_trip(s["x"]), 0, []
        for e, n in enumerate(_counts(case)):
            y = x[at: at + n] @ _exact_values(s["codes"][e], s["scales"][e], case["cols"]).T
            parts.append(y if s["bias"] is None else y + s["bias"][e].double())
            at += n
        return torch.cat(parts)
    out, page, dim = [], case["page"], case["dim"]
    for n in ("k", "v"):
        codes, scales = s[n + "_codes"].flatten(0, 1), s[n + "_scales"].flatten(0, 1)
        if case["format"] == "mx4":
            new = _exact_round_trip(s[n])
        else:
            step = s[n].double().abs().amax(-1, keepdim=True) / 127
            new = torch.where(step > 0, torch.round(s[n].double() / step), 0.0) * step
        place = torch.full((codes.shape[0],), -1, device="cuda", dtype=torch.long)  # which new token a slot got
        place[s["slots"]] = torch.arange(s["slots"].numel(), device="cuda")
        rows = []
        for i, c in enumerate(_contexts(case)):
            at = torch.arange(c, device="cuda")
            slot = s["table"][i].long()[at // page] * page + at % page
            if case["format"] == "mx4":
                held = _exact_values(codes[slot], scales[slot], dim)
            else:
                held = codes[slot].double() * scales[slot].double().unsqueeze(-1)
            rows.append(torch.where((place[slot] >= 0)[:, None, None], new[place[slot].clamp(min=0)], held))
        out.append(torch.cat(rows))
    return out
