"""Rotary positions where there is so much to do that a thread, or a warp, takes several heads: two, four or eight of them, of which a vector
thread has two or four on their way at once; counts that leave a rest, and groups that go from queries to keys."""
import numpy as np
import pytest
import torch

import bounded_cache_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_rotary import BF16, F16, F32, LAYOUTS, NAMES

pytestmark = pytest.mark.gpu


def turned(x, positions, steps, part, pairs, amplitude):
    """bounded_cache_reference.turned for many tokens: [tokens, heads, dim] in 64 bits, and the magnitudes that meet."""
    out, met = x.copy(), np.zeros_like(x)
    with np.errstate(over="ignore"):
        turns = (positions.astype(np.int64)[:, None].view(np.uint64) * steps.view(np.uint64)) / 2.0 ** 64  # whole numbers modulo 2^64
    turns -= np.rint(turns)
    c, s = (amplitude * f(2 * np.pi * turns)[:, None] for f in (np.cos, np.sin))
    half = part // 2
    first, second = (slice(0, part, 2), slice(1, part, 2)) if pairs else (slice(0, half), slice(half, part))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, a * s + b * c
    met[..., first] = met[..., second] = abs(amplitude) * (np.abs(a) + np.abs(b))
    return out, met


def test_the_reference_for_many_tokens_is_the_other_one():
    rng = np.random.default_rng(0)
    x, positions, steps = rng.standard_normal((9, 3, 20)), np.array([0, 1, -1, 5, 1 << 20, 2 ** 31 - 1, -(2 ** 31), 77, 3], np.int32), lce.lce_rotary_steps(16)
    for pairs in (False, True):
        for got, want in zip(turned(x, positions, steps.numpy(), 16, pairs, 1.5), ref.turned(x, positions, steps.tolist(), 16, pairs, 1.5)):
            np.testing.assert_allclose(got, want, rtol=0, atol=1e-13)


def check(got, x, positions, steps, part, layout, amplitude):
    want, met = turned(x.double().cpu().numpy(), positions, steps.numpy(), part, layout == lce.ROTARY_PAIRS, amplitude)
    bound = ref.turned_bound(want, met, NAMES[got.dtype])
    got = got.double().cpu().numpy()
    off = ~(np.abs(got - want) <= bound)
    assert not off.any(), (int(off.sum()), np.abs(got - want)[off].max(), np.argwhere(off)[:5])
    assert np.array_equal(got[..., part:], want[..., part:])


WORK = 148 * 1024  # (token, sixteen channels) times heads that a head more to a thread takes


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("per_thread, q_heads, k_heads", [(2, 13, 3), (2, 5, 0), (4, 9, 1), (4, 6, 11), (8, 13, 3), (8, 9, 1)])
@pytest.mark.parametrize("dim, part, more", [(64, 64, 0), (24, 16, 0), (17, 16, 0), (64, 48, 1)])  # whole vectors in the first two
def test_several_heads_to_a_thread(dtype, layout, per_thread, q_heads, k_heads, dim, part, more):
    units, heads = -(-part // 16) - (-(dim - part) // 16), q_heads + k_heads
    tokens = -(-per_thread * WORK // (units * heads)) + 3
    assert tokens * units * heads < 2 * per_thread * WORK
    rng = np.random.default_rng(tokens)
    stride = heads * dim + more
    wide = torch.from_numpy(rng.standard_normal((tokens, stride), np.float32)).to(dtype).to(DEV)
    before = wide.clone()
    view = lambda t, first, count: t.as_strided((tokens, count, dim), (stride, dim, 1), first * dim)
    positions = rng.integers(-1000, 1 << 20, tokens).astype(np.int32)
    steps = lce.lce_rotary_steps(part)
    desc = lce.make_rotary_desc(dim, part, layout, amplitude=1.25)
    call = lambda q, k, *outs: lce.lce_rotary(desc, q, k, torch.from_numpy(positions).to(DEV), steps.to(DEV), *outs)
    q, k = view(wide, 0, q_heads), view(wide, q_heads, k_heads) if k_heads else None
    out = call(q, k)
    assert torch.equal(wide, before)
    check(out[0], q, positions, steps, part, layout, 1.25)
    if k_heads:
        check(out[1], k, positions, steps, part, layout, 1.25)
    call(q, k, q, k)
    assert torch.equal(q, out[0]) and (not k_heads or torch.equal(k, out[1])) and torch.equal(wide[:, heads * dim:], before[:, heads * dim:])
