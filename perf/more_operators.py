"""Generating with a bounded cache in a binarized transformer: rotary positions, attention weights summed by token, and the
eviction that ranks by them, as cases that can be timed and compared.

A case is a dict of plain values.  Three kinds:

  rotary   queries and keys of new tokens, views into one projection's output, rotated by their positions
  weights  how much attention every token of a 4-bit cache gets from its sequence's newest rows, added to what it had before
  evict    the tokens of each head that had least attention leave the cache, the others move to pages of their own; the rows
           that stay are read back

`own` says which side runs: the plain torch form below, or the library's calls.
"""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32


def _lce():
    import paper_2011_09398_b200
    return paper_2011_09398_b200


# --- cases -------------------------------------------------------------------------------------


def rotary(tokens, q_heads, k_heads, dim, dtype, part=0, layout="halves", scaling="plain", factor=1.0, far=4096, run=True, **more):
    """part: rotated channels of a head (0: all); layout: halves or pairs; scaling: plain, linear, base or parts.
    run: the tokens follow one another (a prompt); otherwise each belongs to a sequence of its own (a decode step).
    far: positions go up to here."""
    return dict(kind="rotary", tokens=tokens, q_heads=q_heads, k_heads=k_heads, dim=dim, dtype=dtype, part=part or dim - dim % 2, layout=layout,
                scaling=scaling, factor=factor, far=far, run=run, **more)


def weights(batch, new, context, kv_heads, group, dim, dtype, page=16, causal=True, window=0, ragged=False, decay=1.0, **more):
    """new: query tokens of each sequence, the last ones of it; context: tokens of the longest sequence, the new ones included;
    decay: what becomes of the weights from before (0: there are none)."""
    return dict(kind="weights", batch=batch, new=new, context=context, kv_heads=kv_heads, group=group, dim=dim, dtype=dtype, page=page,
                causal=causal, window=window, ragged=ragged, decay=decay, **more)


def evict(batch, context, budget, first, recent, kv_heads, dim, dtype, page=16, ragged=False, **more):
    """budget: tokens that a head keeps, the first `first` and the last `recent` among them; dtype: of the rows read back."""
    return dict(kind="evict", batch=batch, new=1, context=context, budget=budget, first=first, recent=recent, kv_heads=kv_heads, dim=dim,
                dtype=dtype, page=page, ragged=ragged, **more)


def listed():
    return [
        # One sequence's decode step, far out: latency.
        rotary(1, 32, 8, 128, "bf16", far=131072, run=False, name="rotary_1_token"),
        # A ragged prompt of a model that rotates part of its heads in neighbouring pairs, fp32 as LceBConv2d writes it.
        rotary(1777, 20, 5, 80, "f32", part=32, layout="pairs", scaling="linear", factor=4.0, name="rotary_1777_d80_f32_pairs"),
        # A long prompt, scaled for a context eight times as long as the model was made for.
        rotary(16384, 32, 8, 128, "bf16", scaling="parts", factor=8.0, far=65536, name="rotary_16384"),
        # One sequence, one new token, a short context: latency.
        weights(1, 1, 777, 8, 4, 128, "bf16", name="weights_b1_777"),
        # A serving batch with contexts of all lengths.
        weights(48, 1, 8192, 8, 4, 128, "bf16", page=64, ragged=True, decay=0.98, name="weights_b48_ragged_8192"),
        # One sequence with a very long context.
        weights(1, 1, 131072, 8, 8, 128, "f16", page=64, name="weights_b1_131072_f16"),
        # fp32 activations, a head for every query head, few queries each (a draft being checked), within a window.
        weights(16, 5, 1500, 12, 1, 64, "f32", window=1024, ragged=True, name="weights_b16_draft5_f32_window"),
        # The last 64 rows of a prompt say what its cache keeps.
        weights(1, 64, 32768, 8, 4, 128, "bf16", page=64, decay=0.0, name="weights_b1_last64_of_32768"),
        # A chunk of a prompt on top of what the cache has.
        weights(2, 1024, 5120, 8, 4, 128, "bf16", page=64, name="weights_b2_prompt1024"),
        # A short sequence that has passed its budget by a page: latency.
        evict(1, 528, 512, 4, 64, 8, 128, "bf16", name="evict_b1_528"),
        # A batch of sequences of all lengths, fp32 rows.
        evict(24, 8192, 2048, 4, 256, 8, 64, "f32", page=64, ragged=True, name="evict_b24_ragged_8192_f32"),
        # One very long prompt cut to a quarter.
        evict(1, 131072, 32768, 16, 1024, 8, 128, "bf16", page=64, name="evict_b1_131072"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _dim(rng):
    return rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]) if rng.random() < 0.8 else rng.randint(17, 255)


def draw(rng):
    kind = rng.choice(["rotary", "rotary", "weights", "weights", "weights", "evict", "evict"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    kv_heads, dim, group = rng.choice([1, 2, 3, 4, 5, 8, 8, 12, 16]), _dim(rng), rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16])
    while True:
        if kind == "rotary":
            part = rng.choice([0, 0, 0, dim // 2 // 2 * 2, 2 * rng.randint(1, dim // 2)])
            case = rotary(_log(rng, 1, 32768), kv_heads * group, kv_heads, dim, dtype, part, rng.choice(["halves", "halves", "pairs"]),
                          rng.choice(["plain", "plain", "linear", "base", "parts"]), rng.choice([2.0, 4.0, 8.0, 32.0]),
                          _log(rng, 64, 1 << 20), run=rng.random() < 0.6)
        elif kind == "weights":
            batch = _log(rng, 1, 64)
            new = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 1024)])
            case = weights(batch, new, new + _log(rng, 1, 65536) - 1, kv_heads, group, dim, dtype, page, causal=rng.random() < 0.8,
                           window=_log(rng, 16, 4096) if rng.random() < 0.2 else 0, ragged=rng.random() < 0.6, decay=rng.choice([0.0, 0.9, 1.0]))
        else:
            batch, context = _log(rng, 1, 48), _log(rng, 1, 131072)
            budget = max(1, int(context * rng.uniform(0.1, 1.1)))
            first = rng.randint(0, min(16, budget))
            case = evict(batch, context, budget, first, rng.randint(0, budget - first) if rng.random() < 0.7 else 0, kv_heads, dim, dtype, page,
                         ragged=rng.random() < 0.6)
        w = work(case)
        if w["bytes"] <= 2.5e8 and w["flops"] <= 7e10 and (kind != "weights" or w["flops"] / (2 * dim) <= 3e8):
            return case


# --- what a pass cannot do without ---------------------------------------------------------------


def _lengths(case):
    """Tokens of each sequence, its new ones included: all the longest, or spread over the range."""
    if not case["ragged"]:
        return [case["context"]] * case["batch"]
    spare = case["context"] - case["new"]
    return [case["context"] if i == 0 else case["new"] + spare * ((i * 7919) % 1009) // 1009 for i in range(case["batch"])]


def _news(case):
    """New tokens of each sequence: fewer of them in some where the batch is ragged."""
    if not case["ragged"]:
        return [case["new"]] * case["batch"]
    return [case["new"] if i % 3 == 0 else 1 + (case["new"] - 1) * ((i * 5087) % 1013) // 1013 for i in range(case["batch"])]


def _visible(case, position, length):
    """First and one past the last token that a query at `position` sees."""
    hi = min(length, position + 1) if case["causal"] else length
    return max(0, position + 1 - case["window"]) if case["window"] else 0, hi


def _row_bytes(case):
    """A key row of one head in the cache: 16 bytes of codes and a scale of 2 for each block; a value row is the same."""
    return ((case["dim"] + BLOCK - 1) // BLOCK) * 18


def _size(case):
    return TYPES[case["dtype"]].itemsize


def work(case):
    if case["kind"] == "rotary":
        rows = case["tokens"] * (case["q_heads"] + case["k_heads"])
        return {"bytes": 2 * rows * case["dim"] * _size(case) + 4 * case["tokens"], "flops": 3 * rows * case["part"]}
    if case["kind"] == "evict":
        tokens, kept = sum(_lengths(case)), sum(min(n, case["budget"]) for n in _lengths(case))
        # scores read; positions and scores of what stays; its rows read, written, read back
        each = 8 + 2 * (3 * _row_bytes(case) + case["dim"] * _size(case))
        return {"bytes": case["kv_heads"] * (4 * tokens + each * kept), "flops": case["kv_heads"] * (tokens + 4 * case["dim"] * kept)}
    heads = case["kv_heads"] * case["group"]
    rows = cached = pairs = 0
    for length, new in zip(_lengths(case), _news(case)):
        lo, _ = _visible(case, length - new, length)
        cached += length - lo
        rows += new
        for i in range(new):
            first, last = _visible(case, length - new + i, length)
            pairs += max(0, last - first)
    outputs = sum(_lengths(case)) * case["kv_heads"] * (8 if case["decay"] else 4)
    return {"bytes": rows * heads * case["dim"] * _size(case) + cached * case["kv_heads"] * _row_bytes(case) + outputs,
            "flops": 2 * pairs * heads * case["dim"]}


# --- inputs ------------------------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _keys_values(g, tokens, case):
    """Keys with channels that stand out, as keys have them; values without; magnitudes that differ between tokens."""
    stand_out = 1 + 7 * (torch.rand(case["kv_heads"], case["dim"], generator=g, device=DEVICE) < 0.05)
    token = torch.exp(0.3 * _normal(g, tokens, 1, 1))
    k = _normal(g, tokens, case["kv_heads"], case["dim"]) * stand_out * 0.7
    v = _normal(g, tokens, case["kv_heads"], case["dim"]) * token
    return k.to(TYPES[case["dtype"]]), v.to(TYPES[case["dtype"]])


def _weights_before(g, *shape):
    """Weights as they add up: a few tokens have most of them, and some have had none."""
    return torch.exp(2 * _normal(g, *shape) - 6) * (torch.rand(shape, generator=g, device=DEVICE) > 0.1)


def _pages_of(case, lengths, seed, order=None):
    """A page table that hands the pages of the pool out in no order: [sequences][most pages], -1 behind the last."""
    counts = [-(-n // case["page"]) for n in lengths]
    if order is None:
        order = list(range(sum(counts) + 1))  # a page more than is used
        random.Random(seed).shuffle(order)
    table, at = [], 0
    for c in counts:
        table.append(order[at:at + c] + [-1] * (max(counts) - c))
        at += c
    return len(order), torch.tensor(table, dtype=torch.int32, device=DEVICE)


def _slots_of(case, table, lengths):
    """The slots of every sequence's tokens, one sequence after the other."""
    parts = []
    for b, n in enumerate(lengths):
        t = torch.arange(n, device=DEVICE)
        parts.append(table[b][t // case["page"]] * case["page"] + t % case["page"])
    return torch.cat(parts).to(torch.int32)


def _inputs(case, seed):
    g = _generator(seed)
    s = {"case": case}
    if case["kind"] == "rotary":
        tokens, dim = case["tokens"], case["dim"]
        wide = _normal(g, tokens, (case["q_heads"] + 2 * case["k_heads"]) * dim).to(TYPES[case["dtype"]])
        s["q"] = wide[:, :case["q_heads"] * dim].view(tokens, -1, dim)
        s["k"] = wide[:, case["q_heads"] * dim:(case["q_heads"] + case["k_heads"]) * dim].view(tokens, -1, dim)
        host = random.Random(seed)
        start = host.randrange(max(1, case["far"] - tokens + 1))
        at = range(start, start + tokens) if case["run"] else [host.randrange(case["far"]) for _ in range(tokens)]
        s["positions"] = torch.tensor(list(at), dtype=torch.int32, device=DEVICE)
        return s
    s["lengths_host"] = _lengths(case)
    s["lengths"] = torch.tensor(s["lengths_host"], dtype=torch.int32, device=DEVICE)
    if case["kind"] == "evict":
        s["kept_host"] = [min(n, case["budget"]) for n in s["lengths_host"]]
        # pages for what there is and for what stays, from one pool
        used = [sum(-(-n // case["page"]) for n in lengths) for lengths in (s["lengths_host"], s["kept_host"])]
        order = list(range(sum(used) + 1))
        random.Random(seed).shuffle(order)
        s["pages"] = len(order)
        s["table"] = _pages_of(case, s["lengths_host"], seed, order)[1]
        s["kept_table"] = _pages_of(case, s["kept_host"], seed, order[used[0]:])[1]
        s["kept_slots"] = _slots_of(case, s["kept_table"], s["kept_host"])
        s["scores"] = _weights_before(g, case["batch"], case["kv_heads"], s["table"].shape[1] * case["page"])
    else:
        s["news_host"] = _news(case)
        s["pages"], s["table"] = _pages_of(case, s["lengths_host"], seed)
        s["q"] = _normal(g, sum(s["news_host"]), case["kv_heads"] * case["group"], case["dim"]).to(TYPES[case["dtype"]])
        starts = [0]
        for n in s["news_host"]:
            starts.append(starts[-1] + n)
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEVICE) if max(s["news_host"]) > 1 else None
        capacity = s["table"].shape[1] * case["page"]
        s["before"] = _weights_before(g, case["batch"], case["kv_heads"], capacity) if case["decay"] else None
        s["out"] = torch.zeros(case["batch"], case["kv_heads"], capacity, device=DEVICE)
    s["slots"] = _slots_of(case, s["table"], s["lengths_host"])
    s["k"], s["v"] = _keys_values(g, s["slots"].numel(), case)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rotary":
        if own:
            lce = _lce()
            layouts = {"halves": lce.ROTARY_HALVES, "pairs": lce.ROTARY_PAIRS}
            scalings = {"plain": lce.ROTARY_PLAIN, "linear": lce.ROTARY_LINEAR, "base": lce.ROTARY_BASE, "parts": lce.ROTARY_PARTS}
            s["desc"] = lce.make_rotary_desc(case["dim"], case["part"], layouts[case["layout"]], amplitude=_amplitude(case))
            s["steps"] = lce.lce_rotary_steps(case["part"], scaling=scalings[case["scaling"]], factor=case["factor"], original_length=ORIGINAL,
                                              low_turns=LOW, high_turns=HIGH).to(DEVICE)
        return s
    if own:
        lce = _lce()
        s["desc"] = lce.make_kv_desc(s["pages"], case["page"], case["kv_heads"], case["dim"])
        s["cache"] = torch.zeros(lce.lce_kv_cache_bytes(s["desc"]), dtype=torch.uint8, device=DEVICE)
        lce.lce_kv_quantize(s["desc"], s["k"], s["v"], s["slots"], s["cache"])
        if case["kind"] == "evict":  # the call wants a table as wide as the budget, also where no sequence has that many tokens
            missing = -(-case["budget"] // case["page"]) - s["kept_table"].shape[1]
            s["kept_table"] = torch.nn.functional.pad(s["kept_table"], (0, max(missing, 0)), value=-1)
    else:
        rows, blocks = s["pages"] * case["page"], (case["dim"] + BLOCK - 1) // BLOCK
        s["cache"] = {name: (torch.zeros(rows, case["kv_heads"], blocks * BLOCK // 2, dtype=torch.uint8, device=DEVICE),
                             torch.zeros(rows, case["kv_heads"], blocks, dtype=torch.bfloat16, device=DEVICE)) for name in "kv"}
        for name in "kv":
            codes, scales = _plain_quantize(s[name])
            s["cache"][name][0][s["slots"].long()] = codes
            s["cache"][name][1][s["slots"].long()] = scales
    del s["k"], s["v"]
    return s


# --- the plain form ------------------------------------------------------------------------------


TOP, ORIGINAL, LOW, HIGH = 10000.0, 8192, 1.0, 32.0  # base of the frequencies, and what the scaling by parts goes by


def _amplitude(case):
    """By which contexts scaled by parts have their queries and keys raised."""
    return 1 + 0.1 * math.log(case["factor"]) if case["scaling"] == "parts" else 1.0


def _frequencies(case):
    """Radians a position turns each pair of channels, in 64 bits."""
    d, factor = case["part"], case["factor"]
    base = TOP
    if case["scaling"] == "base" and d > 2:
        base *= factor ** (d / (d - 2))
    f = [base ** (-2 * i / d) for i in range(d // 2)]
    if case["scaling"] == "linear":
        f = [x / factor for x in f]
    if case["scaling"] == "parts":
        keep = [min(1.0, max(0.0, (ORIGINAL * x / (2 * math.pi) - LOW) / (HIGH - LOW))) for x in f]
        f = [x * (r + (1 - r) / factor) for x, r in zip(f, keep)]
    return torch.tensor(f, dtype=torch.float64, device=DEVICE)


def _plain_rotary(s):
    case = s["case"]
    angle = s["positions"].double()[:, None] * _frequencies(case)
    cos, sin = ((fn(angle) * _amplitude(case)).float()[:, None, :] for fn in (torch.cos, torch.sin))
    half, out = case["part"] // 2, []
    for x in (s["q"], s["k"]):
        x = x.float()
        turned, rest = x[..., :case["part"]], x[..., case["part"]:]
        a, b = (turned[..., :half], turned[..., half:]) if case["layout"] == "halves" else (turned[..., ::2], turned[..., 1::2])
        a, b = a * cos - b * sin, a * sin + b * cos
        turned = torch.cat((a, b), -1) if case["layout"] == "halves" else torch.stack((a, b), -1).flatten(-2)
        out.append(torch.cat((turned, rest), -1).to(TYPES[case["dtype"]]))
    return tuple(out)


def _blocks(x):
    """[rows][heads][dim] -> [rows][heads][blocks][32], zeros behind the last channel."""
    return torch.nn.functional.pad(x, (0, -x.shape[-1] % BLOCK)).unflatten(-1, (-1, BLOCK))


def _plain_quantize(x):
    """Codes two to a byte and scales of a tensor [rows][heads][dim]."""
    x = _blocks(x.float())
    a = x.abs().amax(-1)
    # the smallest bf16 s with 7 s >= a: cut to bf16 from below, one step up where that falls short
    cut = (a.double() / 7).float().view(torch.int32) & -65536
    short = cut.view(torch.float32).double() * 7 < a.double()
    s = torch.where(short, cut + 65536, cut).view(torch.float32)
    codes = torch.where(s[..., None] > 0, torch.round(x.double() / s[..., None].double()), 0.0).to(torch.int32) + 8
    codes = codes.flatten(-2).to(torch.uint8)
    return codes[..., ::2] | (codes[..., 1::2] << 4), s.to(torch.bfloat16)


def _plain_values(codes, scales, dim):
    """fp32 values [rows][heads][dim] that codes and scales stand for."""
    c = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 8
    return (c.unflatten(-1, (-1, BLOCK)) * scales.float()[..., None]).flatten(-2)[..., :dim]


def _plain_weights(s):
    case = s["case"]
    G, H = case["group"], case["kv_heads"]
    out, row = s["out"], 0
    for b, (length, new) in enumerate(zip(s["lengths_host"], s["news_host"])):
        out[b, :, :length] = 0
        if case["decay"]:
            out[b, :, :length - new] = case["decay"] * s["before"][b, :, :length - new]
        lo = _visible(case, length - new, length)[0]
        t = torch.arange(lo, length, device=DEVICE)
        slots = s["table"][b][t // case["page"]].long() * case["page"] + t % case["page"]
        k = _plain_values(*(x[slots] for x in s["cache"]["k"]), case["dim"]).transpose(0, 1)  # [kv heads][tokens][dim]
        q = s["q"][row:row + new].float().view(new, H, G, -1).permute(1, 2, 0, 3).reshape(H, G * new, -1)
        scores = (q @ k.transpose(1, 2) / math.sqrt(case["dim"])).view(H, G, new, -1)
        p = length - new + torch.arange(new, device=DEVICE)[:, None]
        seen = torch.ones(new, t.numel(), dtype=torch.bool, device=DEVICE)
        if case["causal"]:
            seen &= t <= p
        if case["window"]:
            seen &= t > p - case["window"]
        if case["causal"] and new > 1 or case["window"]:
            scores.masked_fill_(~seen, -math.inf)
        e = torch.exp(scores - scores.amax(-1, keepdim=True))
        out[b, :, lo:length] += (e / e.sum(-1, keepdim=True)).sum((1, 2))
        row += new
    return out


def _plain_evict(s):
    case = s["case"]
    B, H, budget, page = case["batch"], case["kv_heads"], case["budget"], case["page"]
    positions = torch.full((B, H, budget), -1, dtype=torch.int32, device=DEVICE)
    scores = torch.zeros(B, H, budget, device=DEVICE)
    head = torch.arange(H, device=DEVICE)
    for b, (n, count) in enumerate(zip(s["lengths_host"], s["kept_host"])):
        rank = s["scores"][b, :, :n].clone()
        if n > budget:
            rank[:, :case["first"]] = math.inf
            rank[:, n - case["recent"]:] = math.inf
        kept = torch.sort(rank, dim=-1, descending=True, stable=True)[1][:, :count].sort(-1)[0]  # [heads][count]
        positions[b, :, :count] = kept
        scores[b, :, :count] = s["scores"][b].gather(1, kept)
        source = s["table"][b][kept // page].long() * page + kept % page
        j = torch.arange(count, device=DEVICE)
        target = s["kept_table"][b][j // page].long() * page + j % page
        for name in "kv":
            for part in s["cache"][name]:
                part[target[:, None], head] = part[source.T, head]
    at = s["kept_slots"].long()
    k, v = (_plain_values(*(x[at] for x in s["cache"][name]), case["dim"]).to(TYPES[case["dtype"]]) for name in "kv")
    return positions, s["lengths"].clamp(max=budget), scores, k, v


# --- one pass ------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if not own:
        return {"rotary": _plain_rotary, "weights": _plain_weights, "evict": _plain_evict}[case["kind"]](s)
    lce = _lce()
    if case["kind"] == "rotary":
        return lce.lce_rotary(s["desc"], s["q"], s["k"], s["positions"], s["steps"])
    if case["kind"] == "weights":
        return lce.lce_kv_attention_weights(s["desc"], s["q"], s["cache"], s["table"], s["lengths"], s["q_starts"], causal=case["causal"],
                                            window=case["window"], previous=s["before"], decay=case["decay"], out=s["out"])
    kept = lce.lce_kv_evict(s["desc"], s["cache"], s["table"], s["lengths"], s["scores"], s["kept_table"], case["budget"], first=case["first"],
                            recent=case["recent"])
    return kept + lce.lce_kv_dequantize(s["desc"], s["cache"], s["kept_slots"], TYPES[case["dtype"]])


# --- the definitions in 64 bits ------------------------------------------------------------------


def _exact_quantized(x):
    """Values that the rows of x stand for once they are stored, block by block of 32 channels."""
    x = x.double()
    out = torch.zeros_like(x)
    for c in range(0, x.shape[-1], 32):
        part = x[..., c:c + 32]
        mantissa, exponent = torch.frexp(part.abs().amax(-1, keepdim=True) / 7)
        step = torch.ldexp(torch.ceil(mantissa * 256) / 256, exponent)  # eight significant bits, upwards
        out[..., c:c + 32] = torch.where(step > 0, torch.round(part / torch.where(step > 0, step, 1.0)), 0.0) * step
    return out


def _exact_rotary(s):
    case = s["case"]
    d, factor = case["part"], case["factor"]
    i = torch.arange(d // 2, dtype=torch.float64, device=DEVICE)
    exponent = math.log(TOP) + (math.log(factor) * d / (d - 2) if case["scaling"] == "base" and d > 2 else 0.0)
    f = torch.exp(-2 * i / d * exponent)
    if case["scaling"] == "linear":
        f = f / factor
    if case["scaling"] == "parts":
        ramp = torch.clamp((ORIGINAL / (2 * math.pi) * f - LOW) / (HIGH - LOW), 0, 1)
        f = torch.lerp(f / factor, f, ramp)
    turn = _amplitude(case) * torch.exp(1j * s["positions"].double()[:, None, None] * f)
    out = []
    for x in (s["q"], s["k"]):
        x = x.double().clone()
        part = x[..., :d]
        first, second = (slice(0, d // 2), slice(d // 2, d)) if case["layout"] == "halves" else (slice(0, d, 2), slice(1, d, 2))
        z = torch.complex(part[..., first].contiguous(), part[..., second].contiguous()) * turn
        part[..., first], part[..., second] = z.real, z.imag
        out.append(x)
    return tuple(out)


def _exact_evict(s):
    case = s["case"]
    positions, scores, rows = [], [], {"k": [], "v": []}
    token = 0
    values = {name: _exact_quantized(s[name]) for name in "kv"}
    for b, n in enumerate(s["lengths_host"]):
        for h in range(case["kv_heads"]):
            have = s["scores"][b, h, :n].double().cpu().numpy()
            keep = np.arange(n)
            if n > case["budget"]:
                others = keep[case["first"]:n - case["recent"]]
                best = others[np.lexsort((others, -have[others]))[:case["budget"] - case["first"] - case["recent"]]]
                keep = np.sort(np.concatenate([keep[:case["first"]], best, keep[n - case["recent"]:]]))
            spare = case["budget"] - len(keep)
            positions.append(np.pad(keep, (0, spare), constant_values=-1))
            scores.append(np.pad(have[keep], (0, spare)))
            for name in "kv":
                rows[name].append(values[name][token + torch.from_numpy(keep).to(DEVICE), h])
        token += n
    H = case["kv_heads"]
    out = [torch.cat([torch.stack(rows[name][b * H:(b + 1) * H], 1) for b in range(case["batch"])]) for name in "kv"]
    shape = (case["batch"], H, case["budget"])
    return (torch.from_numpy(np.stack(positions)).to(DEVICE, torch.int32).view(shape), torch.tensor(s["kept_host"], dtype=torch.int32, device=DEVICE),
            torch.from_numpy(np.stack(scores)).to(DEVICE).view(shape), *out)


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "rotary":
        return _exact_rotary(s)
    if case["kind"] == "evict":
        return _exact_evict(s)
    k = _exact_quantized(s["k"])
    out = torch.zeros(case["batch"], case["kv_heads"], s["table"].shape[1] * case["page"], dtype=torch.float64, device=DEVICE)
    token = row = 0
    for b, (length, new) in enumerate(zip(s["lengths_host"], s["news_host"])):
        place, at = torch.arange(length, device=DEVICE), torch.arange(length - new, length, device=DEVICE)[:, None]
        for h in range(case["kv_heads"] * case["group"]):
            score = s["q"][row:row + new, h].double() @ k[token:token + length, h // case["group"]].T * case["dim"] ** -0.5
            if case["causal"]:
                score = torch.where(place > at, -math.inf, score)
            if case["window"]:
                score = torch.where(place <= at - case["window"], -math.inf, score)
            out[b, h // case["group"], :length] += torch.softmax(score, -1).sum(0)
        if case["decay"]:
            out[b, :, :length - new] += case["decay"] * s["before"][b, :, :length - new].double()
        token, row = token + length, row + new
    return out
