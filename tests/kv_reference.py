"""The operators between binary projections written down in 64 bits, without the library: what its tests compare with."""
import numpy as np

HALF_STEP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}  # largest relative rounding of each type


def quantized(x):
    """Values and scales that float64 rows [..., dim] stand for in the cache: blocks of 32 channels, the scale the smallest number
    of eight significant bits (bf16) with 7 s >= max |x|, codes rounded half to even; NaN throughout a block that is not finite."""
    x = np.asarray(x, np.float64)
    out, scales = np.zeros_like(x), []
    for c in range(0, x.shape[-1], 32):
        part = x[..., c:c + 32]
        with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
            top = np.abs(part).max(-1, keepdims=True)
            bad = ~np.isfinite(top)
            mantissa, exponent = np.frexp(np.where(bad, 1.0, top) / 7)
            # bf16 numbers below 2^-126 are the multiples of 2^-133
            step = np.ldexp(1.0, np.maximum(exponent - 8, -133))
            s = np.ceil(np.ldexp(mantissa, exponent) / step) * step
            codes = np.where(s > 0, np.rint(np.where(bad, 0.0, part) / np.where(s > 0, s, 1.0)), 0.0)
        out[..., c:c + 32] = np.where(bad, np.nan, codes * s)
        scales.append(np.where(bad, np.nan, s)[..., 0])
    return out, np.stack(scales, -1)


def attention(q, k, v, k_scales, v_scales, shown, scale, rows_type):
    """Rows q [heads][dim] of one position against keys and values [tokens][kv heads][dim]: the result in 64 bits and how far the
    library's may be off.  shown: bool [tokens].

    The bound, per channel: half a step of the output's type; weights rounded to f16 (2^-11 each; as two f16 numbers for fp32
    rows: 2^-21), 2^-31 of the largest value for a weight too small for f16; fp32 sums over the tokens, one step (2^-23, they may be
    cut) for each of the at most ceil(tokens / 16) products and 64 steps for joining warps and pieces, the exponentials and the
    quotient; and the scores' own error e, by which a weight moves by the factor 1 +- e and their sum by as much: their sums are
    of at most 15 s |q| per channel, in 6 steps.  16-bit rows have codes as subnormal numbers n 2^-22 for operands: a product adds up
    17 terms cut at 2^-23 of what its largest exponents allow, 2^-14 |q| (not 2^-22 |q|): 17 * 2^-15 of a code's step and the largest
    |q| for each of a block's two products, and of the largest weight for each of a tile's two.  (Many rows have keys and values as f16
    numbers c s for operands, exact down to 2^-28 of the largest scale of 128 tokens; below, off by 2^-39 of the largest value.)"""
    heads, group = q.shape[0], q.shape[0] // k.shape[1]
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    if not shown.any():
        return out, bound
    at = np.flatnonzero(shown)
    for h in range(heads):
        kk, vv = k[at, h // group], v[at, h // group]
        with np.errstate(invalid="ignore", over="ignore"):
            s = kk @ q[h] * scale
            w = np.exp(s - s.max())
            w /= w.sum()
            out[h] = w @ vv
            per_channel = np.repeat(k_scales[at, h // group], 32, -1)[:, :q.shape[1]]
            e = 6 * 2.0 ** -23 * 15 * abs(scale) * (per_channel * np.abs(q[h])).sum(-1).max()
            e += 2.0 ** -23 * np.abs(s - s.max()).max() * 1.5  # the argument of the exponential
            cut = 0.0
            if rows_type != "float32":
                e += 34 * 2.0 ** -15 * abs(scale) * np.abs(q[h]).max() * k_scales[at, h // group].sum(-1).max()
                cut = 34 * 2.0 ** -15 * np.repeat(w @ np.nan_to_num(v_scales[at, h // group]), 32)[:q.shape[1]]
                cut = cut + 2.0 ** -39 * np.nan_to_num(np.abs(vv), nan=0.0).max()
            weight = (2.0 ** -11 if rows_type != "float32" else 2.0 ** -21) + 2 * e + (len(at) // 16 + 65) * 2.0 ** -23
            bound[h] = HALF_STEP[rows_type] * np.abs(out[h]) + cut + weight * (w @ np.abs(vv)) + 2.0 ** -31 * len(at) * np.nan_to_num(np.abs(vv), nan=0.0).max()
    return out, bound


def normed(v, kind, weight, bias, eps):
    if kind == "layer":
        v = v - v.mean(-1, keepdims=True)
    if kind != "none":
        v = v / np.sqrt((v * v).mean(-1, keepdims=True) + eps)
    if weight is not None:
        v = v * weight.astype(np.float64)
    if bias is not None:
        v = v + bias.astype(np.float64)
    return v


def packed(z):
    bits = np.zeros(z.shape[:-1] + (-(-z.shape[-1] // 32) * 32,), np.uint64)
    bits[..., :z.shape[-1]] = z < 0
    return (bits.reshape(z.shape[:-1] + (-1, 32)) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32)
