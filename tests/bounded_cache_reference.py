"""Rotary positions, attention weights by token and eviction written down in 64 bits, without the library: what their tests compare with."""
import numpy as np

import kv_reference as ref

HALF_STEP = ref.HALF_STEP


def turned(x, positions, steps, rotary_dim, pairs, amplitude):
    """Rows x [tokens, heads, dim] by their positions and steps (units of 2^-64 turns): the result in 64 bits and, element by element, the
    sum of the magnitudes that meet in it."""
    x = np.asarray(x, np.float64)
    out, met = x.copy(), np.zeros_like(x)
    for t, position in enumerate(positions):
        part = np.array([(int(position) * int(s)) % (1 << 64) / 2.0 ** 64 for s in steps])  # whole numbers: exact
        part -= np.rint(part)
        c, s = amplitude * np.cos(2 * np.pi * part), amplitude * np.sin(2 * np.pi * part)
        half = rotary_dim // 2
        at = (slice(0, rotary_dim, 2), slice(1, rotary_dim, 2)) if pairs else (slice(0, half), slice(half, rotary_dim))
        a, b = x[t][:, at[0]], x[t][:, at[1]]
        out[t][:, at[0]], out[t][:, at[1]] = a * c - b * s, a * s + b * c
        met[t][:, at[0]] = met[t][:, at[1]] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return out, met


def turned_bound(out, met, dtype):
    """Angles off by 2^-33 of a turn and by 2^-25 of themselves (at most an eighth of a turn), the sums by 2^-28: sines and cosines are off by
    2^-23.  The amplitude, two products and a sum of fp32 are four roundings of 2^-24: 2^-22 more of the magnitudes that meet.  Then
    half a step of the output's type (fp16 and bf16 numbers below the normal ones: of the smallest normal)."""
    least = {"float32": 2.0 ** -126, "float16": 2.0 ** -14, "bfloat16": 2.0 ** -126}[dtype]
    return (2.0 ** -23 + 2.0 ** -22) * met + HALF_STEP[dtype] * np.maximum(np.abs(out), np.where(met > 0, least, 0.0)) * (1 + 2.0 ** -20)


def weights(q, k, k_scales, shown, scale):
    """Weights that rows q [rows, heads, dim] of one sequence give its tokens (keys [tokens, kv heads, dim] as the cache holds them), summed by
    kv head: [kv heads, tokens], and how far the library's may be off.  shown: bool [rows, tokens].

    The bound: a score is a sum of at most 15 s |q| per channel in steps of 2^-23, six of them at most for the block's products (fp32 rows: of
    22 bits), its scale and the sum over blocks; the factor and the difference from the largest round to 2^-24 of themselves each.  A weight moves by as
    much, and so does their sum: twice that.  Sums over tokens: one step for each of a lane's tokens (every 16th at most) and 64 for exponentials,
    joining and the quotient.  Then the sum over the columns, a step for each."""
    rows, heads, _ = q.shape
    kv_heads, tokens = k.shape[1], k.shape[0]
    out, bound = np.zeros((kv_heads, tokens)), np.zeros((kv_heads, tokens))
    group = heads // kv_heads
    for h in range(heads):
        kk = k[:, h // group]
        per_channel = np.repeat(k_scales[:, h // group], 32, -1)[:, :q.shape[2]]
        for i in range(rows):
            at = np.flatnonzero(shown[i])
            if not len(at):
                continue
            with np.errstate(invalid="ignore", over="ignore"):
                s = kk[at] @ q[i, h] * scale
                w = np.exp(s - s.max())
                w /= w.sum()
                e = 6 * 2.0 ** -23 * 15 * abs(scale) * (per_channel[at] * np.abs(q[i, h])).sum(-1).max()
                e += 2.0 ** -23 * (np.abs(s).max() + np.abs(s - s.max()).max())
                out[h // group, at] += w
                bound[h // group, at] += w * (2 * e + (len(at) // 16 + 65) * 2.0 ** -23) + 2.0 ** -125
    return out, bound + (rows * group + 4) * 2.0 ** -24 * np.abs(out)


def kept(scores, n, valid, budget, first, recent):
    """The places among n tokens that a head keeps, ascending.  scores [n], valid bool [n]."""
    places = np.arange(n)
    if n <= budget:
        return places[valid[:n]]
    always = (places < first) | (places >= n - recent)
    s = np.asarray(scores[:n], np.float64) + 0.0
    # highest first: what is always kept, numbers, NaN; ties to the earlier
    level = np.where(always, 2, np.where(np.isnan(s), 0, 1))
    s = np.where(np.isnan(s) | always, 0.0, s)
    order = np.lexsort((places, -s, -level))
    order = order[valid[order]]
    return np.sort(order[:budget])
