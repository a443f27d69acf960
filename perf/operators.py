"""The operators between the projections of a binarized transformer, as cases that can be timed and compared.

A case is a dict of plain values.  Four kinds:

  store      keys and values of new tokens quantised into a 4-bit cache (blocks of 32 channels, a bf16 scale each,
             codes -7 .. 7) at the slots they are given, and the rows that were stored read back
  load       rows of a filled cache read back by their slots, in whatever order the page table has them
  attention  queries of one or more new tokens of each sequence against the sequence's pages of the cache
  norm       the norm behind a block, its gate and residual scale, the residual add, the norm in front of the next
             block and, where that block's projections are binarized, the sign bits of its result

`own` says which side runs: the plain torch form below, or the library's calls.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEVICE = "cuda:0"
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BLOCK = 32
EPS, SCALE = 2.0 ** -17, 0.75  # of the norms and of the residual add; both fp32 values


def _lce():
    import paper_2011_09398_b200
    return paper_2011_09398_b200


# --- cases -------------------------------------------------------------------------------------


def store(tokens, kv_heads, dim, dtype, page=16, strided=False, run=True, **more):
    """run: the tokens follow one another in their pages (a prompt); otherwise each has a page of its own (a decode step).
    strided: k and v are views into one projection's output."""
    return dict(kind="store", tokens=tokens, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, strided=strided, run=run, **more)


def load(tokens, kv_heads, dim, dtype, page=16, **more):
    return dict(kind="load", tokens=tokens, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, **more)


def attention(batch, new, context, kv_heads, group, dim, dtype, page=16, causal=True, window=0, ragged=False, **more):
    """new: query tokens of each sequence, the last ones of it; context: tokens of the longest sequence, the new ones included."""
    return dict(kind="attention", batch=batch, new=new, context=context, kv_heads=kv_heads, group=group, dim=dim, dtype=dtype,
                page=page, causal=causal, window=window, ragged=ragged, **more)


def norm(rows, channels, dtype, stream, post, pre, gate="none", out="normed", **more):
    """dtype: of the block's output, its gate and the normed result; stream: of the residual stream.
    gate: none, plain (values as they are) or sigmoid.  out: normed, bits or both."""
    return dict(kind="norm", rows=rows, channels=channels, dtype=dtype, stream=stream, post=post, pre=pre, gate=gate, out=out, **more)


def listed():
    return [
        # One sequence's decode step: one token goes into the cache.
        store(1, 8, 128, "bf16", run=False, name="store_1_token"),
        # A model whose heads are not whole blocks and whose projection writes q, k and v side by side in fp32, as
        # LceBConv2d does: a ragged prompt.
        store(1777, 5, 80, "f32", strided=True, name="store_1777_d80_f32_strided"),
        # A long prompt.
        store(16384, 8, 128, "bf16", name="store_16384_prompt"),
        # A short history goes back to full precision for a layer that wants it so.
        load(500, 8, 64, "f32", name="load_500_d64_f32"),
        # A long one.
        load(32768, 8, 128, "bf16", page=64, name="load_32768"),
        # One sequence, one new token, a short context: latency.
        attention(1, 1, 777, 8, 4, 128, "bf16", name="attention_b1_777"),
        # A serving batch with contexts of all lengths.
        attention(48, 1, 8192, 8, 4, 128, "bf16", page=64, ragged=True, name="attention_b48_ragged_8192"),
        # One sequence with a very long context.
        attention(1, 1, 131072, 8, 8, 128, "f16", page=64, name="attention_b1_131072_f16"),
        # fp32 activations, a head for every query head, few queries each (a draft being checked), within a window.
        attention(16, 5, 1500, 12, 1, 64, "f32", window=1024, ragged=True, name="attention_b16_draft5_f32_window"),
        # A chunk of a prompt on top of what the cache has.
        attention(2, 1024, 5120, 8, 4, 128, "bf16", page=64, name="attention_b2_prompt1024"),
        # One token's row through a block boundary: latency.
        norm(1, 4096, "bf16", "bf16", "rms", "rms", gate="sigmoid", name="norm_1_4096"),
        # A prompt's rows, fp32 residual stream, bits for the next binary projections.
        norm(8000, 4000, "f32", "f32", "layer", "layer", gate="plain", out="bits", name="norm_8000_4000_f32_bits"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _dim(rng):
    return rng.choice([64, 64, 80, 96, 128, 128, 128, 192, 256]) if rng.random() < 0.8 else rng.randint(17, 255)


def draw(rng):
    kind = rng.choice(["store", "load", "attention", "attention", "attention", "norm", "norm"])
    dtype = rng.choice(["f32", "f16", "bf16", "bf16"])
    page = rng.choice([16, 16, 32, 48, 64, 128])
    if kind == "norm":
        channels = _log(rng, 64, 16384)
        if rng.random() < 0.7:
            channels = max(64, channels // 32 * 32)
        rows = _log(rng, 1, max(1, min(16384, 32_000_000 // channels)))
        pre = rng.choice(["rms", "layer"])
        return norm(rows, channels, dtype, rng.choice([dtype, "f32"]), rng.choice(["none", "rms", "layer"]), pre,
                    rng.choice(["none", "plain", "sigmoid"]), rng.choice(["normed", "bits", "both"]))
    kv_heads, dim = rng.choice([1, 2, 3, 4, 5, 8, 8, 12, 16]), _dim(rng)
    if kind != "attention":
        tokens = _log(rng, 1, max(1, min(32768, 16384 * 8 * 128 // (kv_heads * dim))))
        if kind == "load":
            return load(tokens, kv_heads, dim, dtype, page)
        return store(tokens, kv_heads, dim, dtype, page, strided=rng.random() < 0.4, run=tokens > 512 or rng.random() < 0.5)
    while True:
        batch = _log(rng, 1, 64)
        new = rng.choice([1, 1, 1, rng.randint(2, 8), _log(rng, 9, 1024)])
        case = attention(batch, new, new + _log(rng, 1, 65536) - 1, kv_heads, rng.choice([1, 1, 2, 3, 4, 4, 7, 8, 16]), dim, dtype, page,
                         causal=rng.random() < 0.8, window=_log(rng, 16, 4096) if rng.random() < 0.2 else 0, ragged=rng.random() < 0.6)
        w = work(case)
        if w["flops"] <= 1.2e11 and w["bytes"] <= 1.5e8:
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
    """A key and a value row of one head in the cache: 16 bytes of codes and a scale of 2 for each block."""
    return 2 * ((case["dim"] + BLOCK - 1) // BLOCK) * 18


def _size(dtype):
    return TYPES[dtype].itemsize


def work(case):
    if case["kind"] == "norm":
        n = case["rows"] * case["channels"]
        wide = 2 * _size(case["stream"]) + _size(case["dtype"]) * (1 + (case["gate"] != "none") + (case["out"] != "bits"))
        return {"bytes": n * wide + (n // 8 if case["out"] != "normed" else 0), "flops": 20 * n}
    if case["kind"] in ("store", "load"):
        values = 2 * case["tokens"] * case["kv_heads"] * case["dim"]
        cached = case["tokens"] * case["kv_heads"] * _row_bytes(case)
        times = 2 if case["kind"] == "store" else 1  # stored, then read back
        return {"bytes": times * (values * _size(case["dtype"]) + cached), "flops": times * 4 * values}
    heads = case["kv_heads"] * case["group"]
    tokens = cached = pairs = 0
    for length, new in zip(_lengths(case), _news(case)):
        lo, _ = _visible(case, length - new, length)
        cached += max(0, length - lo)
        tokens += new
        for i in range(new):
            first, last = _visible(case, length - new + i, length)
            pairs += max(0, last - first)
    return {"bytes": 2 * tokens * heads * case["dim"] * _size(case["dtype"]) + cached * case["kv_heads"] * _row_bytes(case),
            "flops": 4 * pairs * heads * case["dim"]}


# --- inputs ------------------------------------------------------------------------------------


def _generator(seed):
    return torch.Generator(device=DEVICE).manual_seed(seed)


def _normal(g, *shape):
    return torch.randn(shape, generator=g, device=DEVICE)


def _keys_values(g, tokens, kv_heads, dim, dtype):
    """Keys with channels that stand out, as keys have them; values without; magnitudes that differ between tokens."""
    stand_out = 1 + 7 * (torch.rand(kv_heads, dim, generator=g, device=DEVICE) < 0.05)
    token = torch.exp(0.3 * _normal(g, tokens, 1, 1))
    k = _normal(g, tokens, kv_heads, dim) * stand_out * 0.7
    v = _normal(g, tokens, kv_heads, dim) * token
    return k.to(TYPES[dtype]), v.to(TYPES[dtype])


def _pages_of(case, lengths, seed):
    """A page table that hands the pages of the pool out in no order: [sequences][most pages], -1 behind the last."""
    counts = [-(-n // case["page"]) for n in lengths]
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
    if case["kind"] == "norm":
        shape, dtype = (case["rows"], case["channels"]), TYPES[case["dtype"]]
        s["x"] = (2 * _normal(g, *shape)).to(TYPES[case["stream"]])
        s["branch"] = (_normal(g, *shape) * torch.exp(0.5 * _normal(g, shape[0], 1))).to(dtype)
        s["gate"] = _normal(g, *shape).to(dtype) if case["gate"] != "none" else None
        for name, kind in (("post", case["post"]), ("pre", case["pre"])):
            s[name + "_weight"] = 1 + 0.2 * _normal(g, shape[1]) if kind != "none" else None
            s[name + "_bias"] = 0.1 * _normal(g, shape[1]) if kind == "layer" else None
        return s
    if case["kind"] == "attention":
        s["lengths_host"], s["news_host"] = _lengths(case), _news(case)
        s["pages"], s["table"] = _pages_of(case, s["lengths_host"], seed)
        s["slots"] = _slots_of(case, s["table"], s["lengths_host"])
        s["k"], s["v"] = _keys_values(g, s["slots"].numel(), case["kv_heads"], case["dim"], case["dtype"])
        s["q"] = _normal(g, sum(s["news_host"]), case["kv_heads"] * case["group"], case["dim"]).to(TYPES[case["dtype"]])
        s["lengths"] = torch.tensor(s["lengths_host"], dtype=torch.int32, device=DEVICE)
        starts = [0]
        for n in s["news_host"]:
            starts.append(starts[-1] + n)
        s["q_starts"] = torch.tensor(starts, dtype=torch.int32, device=DEVICE) if max(s["news_host"]) > 1 else None
        return s
    tokens, H, D = case["tokens"], case["kv_heads"], case["dim"]
    if case["kind"] == "store" and not case["run"]:
        s["pages"] = tokens + 1
        order = list(range(s["pages"]))
        random.Random(seed).shuffle(order)
        offset = random.Random(seed + 1)
        s["slots"] = torch.tensor([p * case["page"] + offset.randrange(case["page"]) for p in order[:tokens]], dtype=torch.int32, device=DEVICE)
    else:
        s["pages"], table = _pages_of(case, [tokens], seed)
        s["slots"] = _slots_of(case, table, [tokens])
    s["k"], s["v"] = _keys_values(g, tokens, H, D, case["dtype"])
    if case.get("strided"):
        wide = torch.zeros(tokens, 3 * H * D + 8, dtype=TYPES[case["dtype"]], device=DEVICE)
        views = [wide[:, H * D + i * H * D:H * D + (i + 1) * H * D].view(tokens, H, D) for i in range(2)]
        views[0].copy_(s["k"])
        views[1].copy_(s["v"])
        s["k"], s["v"] = views
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "norm":
        if own:
            lce = _lce()
            norms = {"none": lce.NORM_NONE, "rms": lce.NORM_RMS, "layer": lce.NORM_LAYER}
            s["desc"] = lce.make_norm_desc(case["rows"], case["channels"], norms[case["post"]], norms[case["pre"]], eps=EPS, residual_scale=SCALE,
                                           gate_activation=lce.ACT_SIGMOID if case["gate"] == "sigmoid" else lce.ACT_NONE)
        return s
    if own:
        lce = _lce()
        s["desc"] = lce.make_kv_desc(s["pages"], case["page"], case["kv_heads"], case["dim"])
        s["cache"] = torch.zeros(lce.lce_kv_cache_bytes(s["desc"]), dtype=torch.uint8, device=DEVICE)
    else:
        rows, blocks = s["pages"] * case["page"], (case["dim"] + BLOCK - 1) // BLOCK
        s["cache"] = {name: (torch.zeros(rows, case["kv_heads"], blocks * BLOCK // 2, dtype=torch.uint8, device=DEVICE),
                             torch.zeros(rows, case["kv_heads"], blocks, dtype=torch.bfloat16, device=DEVICE)) for name in "kv"}
    if case["kind"] != "store":
        if own:
            _lce().lce_kv_quantize(s["desc"], s["k"], s["v"], s["slots"], s["cache"])
        else:
            _plain_store(s)
        del s["k"], s["v"]
    if case["kind"] == "load":  # read back from the end to the start, as no program stores it
        s["slots"] = s["slots"].flip(0).contiguous()
    return s


# --- the plain form ------------------------------------------------------------------------------


def _blocks(x):
    """[rows][heads][dim] -> [rows][heads][blocks][32], zeros behind the last channel."""
    pad = -x.shape[-1] % BLOCK
    return torch.nn.functional.pad(x, (0, pad)).unflatten(-1, (-1, BLOCK))


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


def _plain_store(s):
    at = s["slots"].long()
    for name in "kv":
        codes, scales = _plain_quantize(s[name])
        s["cache"][name][0][at] = codes
        s["cache"][name][1][at] = scales


def _plain_load(s, name, slots):
    codes, scales = s["cache"][name]
    return _plain_values(codes[slots], scales[slots], s["case"]["dim"])


def _plain_attention(s):
    case = s["case"]
    G, H = case["group"], case["kv_heads"]
    out, row = torch.empty_like(s["q"]), 0
    for b, (length, new) in enumerate(zip(s["lengths_host"], s["news_host"])):
        lo = _visible(case, length - new, length)[0]
        t = torch.arange(lo, length, device=DEVICE)
        slots = s["table"][b][t // case["page"]].long() * case["page"] + t % case["page"]
        k, v = (_plain_load(s, name, slots).transpose(0, 1) for name in "kv")  # [kv heads][tokens][dim]
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
        o = (e.view(H, G * new, -1) @ v).view(H, G, new, -1) / e.sum(-1, keepdim=True)
        out[row:row + new] = o.permute(2, 0, 1, 3).reshape(new, H * G, -1)
        row += new
    return out


def _plain_norm_of(v, kind):
    if kind == "rms":
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    if kind == "layer":
        v = v - v.mean(-1, keepdim=True)
        return v * torch.rsqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v


def _plain_bits(z):
    """bit = (z < 0), 32 channels to a word, zeros behind the last channel."""
    bits = _blocks((z < 0).to(torch.int64)) << torch.arange(BLOCK, device=DEVICE)
    return bits.sum(-1).to(torch.int32)


def _plain_norm(s):
    case = s["case"]
    wide = torch.float64 if case["out"] != "normed" else torch.float32  # signs next to zero
    u = _plain_norm_of(s["branch"].to(wide), case["post"])
    if case["post"] != "none":
        u = u * s["post_weight"]
    if case["post"] == "layer":
        u = u + s["post_bias"]
    u = u * SCALE
    if s["gate"] is not None:
        gate = s["gate"].to(wide)
        u = u * (1 / (1 + torch.exp(-gate)) if case["gate"] == "sigmoid" else gate)
    y = s["x"].to(wide) + u
    z = _plain_norm_of(y, case["pre"]) * s["pre_weight"]
    if case["pre"] == "layer":
        z = z + s["pre_bias"]
    out = {"y": y.to(TYPES[case["stream"]])}
    if case["out"] != "bits":
        out["normed"] = z.to(TYPES[case["dtype"]])
    if case["out"] != "normed":
        out["bits"] = _plain_bits(z)
    return out


# --- one pass ------------------------------------------------------------------------------------


def run(s):
    case = s["case"]
    if not own:
        if case["kind"] == "norm":
            return _plain_norm(s)
        if case["kind"] == "attention":
            return _plain_attention(s)
        if case["kind"] == "store":
            _plain_store(s)
        return tuple(_plain_load(s, name, s["slots"].long()).to(TYPES[case["dtype"]]) for name in "kv")
    lce = _lce()
    if case["kind"] == "norm":
        y = torch.empty_like(s["x"])
        normed = torch.empty_like(s["branch"]) if case["out"] != "bits" else None
        bits = torch.empty(case["rows"], (case["channels"] + 31) // 32, dtype=torch.int32, device=DEVICE) if case["out"] != "normed" else None
        lce.lce_residual_norm(s["desc"], s["x"], s["branch"], s["gate"], s["post_weight"], s["post_bias"], s["pre_weight"], s["pre_bias"],
                              y, normed, bits)
        return {name: t for name, t in (("y", y), ("normed", normed), ("bits", bits)) if t is not None}
    if case["kind"] == "attention":
        return lce.lce_kv_attention(s["desc"], s["q"], s["cache"], s["table"], s["lengths"], s["q_starts"], causal=case["causal"],
                                    window=case["window"])
    if case["kind"] == "store":
        lce.lce_kv_quantize(s["desc"], s["k"], s["v"], s["slots"], s["cache"])
    return lce.lce_kv_dequantize(s["desc"], s["cache"], s["slots"], TYPES[case["dtype"]])


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


def exact(case, seed):
    s = _inputs(case, seed)
    if case["kind"] == "norm":
        def normed(v, kind, w, b):
            if kind == "none":
                return v
            if kind == "layer":
                v = v - v.sum(-1, keepdim=True) / v.shape[-1]
            v = v / torch.sqrt(v.square().sum(-1, keepdim=True) / v.shape[-1] + EPS) * w.double()
            return v if b is None else v + b.double()
        factor = torch.full_like(s["x"], SCALE, dtype=torch.float64)
        if case["gate"] != "none":
            factor = factor * (torch.sigmoid(s["gate"].double()) if case["gate"] == "sigmoid" else s["gate"].double())
        y = s["x"].double() + factor * normed(s["branch"].double(), case["post"], s["post_weight"], s["post_bias"])
        z = normed(y, case["pre"], s["pre_weight"], s["pre_bias"])
        out = {"y": y}
        if case["out"] != "bits":
            out["normed"] = z
        if case["out"] != "normed":
            words = torch.zeros(z.shape[0], -(-z.shape[1] // 32), dtype=torch.int64, device=DEVICE)
            for c in range(32):
                column = (z[:, c::32] < 0).long() << c
                words[:, :column.shape[1]] += column
            out["bits"] = torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)
        return out
    k, v = _exact_quantized(s["k"]), _exact_quantized(s["v"])
    if case["kind"] == "load":
        return k.flip(0), v.flip(0)
    if case["kind"] == "store":
        return k, v
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    token = row = 0
    for length, new in zip(s["lengths_host"], s["news_host"]):
        for h in range(out.shape[1]):
            keys, values = k[token:token + length, h // case["group"]], v[token:token + length, h // case["group"]]
            score = s["q"][row:row + new, h].double() @ keys.T * case["dim"] ** -0.5
            place, at = torch.arange(length, device=DEVICE), torch.arange(length - new, length, device=DEVICE)[:, None]
            if case["causal"]:
                score = torch.where(place > at, -math.inf, score)
            if case["window"]:
                score = torch.where(place <= at - case["window"], -math.inf, score)
            out[row:row + new, h] = torch.softmax(score, -1) @ values
        token, row = token + length, row + new
    return out
