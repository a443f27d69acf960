"""Rotary positions against the definition in 64 bits; bounded_cache_reference.turned_bound derives the bounds."""
import numpy as np
import pytest
import torch

import bounded_cache_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV

pytestmark = pytest.mark.gpu
NAMES = {torch.float32: "float32", torch.float16: "float16", torch.bfloat16: "bfloat16"}
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
LAYOUTS = [lce.ROTARY_HALVES, lce.ROTARY_PAIRS]


def rows(rng, dtype, tokens, heads, dim, more=0):
    """[tokens, heads, dim] in a buffer whose rows are `more` elements longer."""
    wide = torch.from_numpy(rng.standard_normal((tokens, heads * dim + more))).to(dtype).to(DEV)
    return wide[:, :heads * dim].view(tokens, heads, dim) if not more else wide.as_strided((tokens, heads, dim), (heads * dim + more, dim, 1))


def check(got, x, positions, steps, rotary_dim, layout, amplitude=1.0):
    want, met = ref.turned(x.double().cpu().numpy(), positions, steps.tolist(), rotary_dim, layout == lce.ROTARY_PAIRS, amplitude)
    bound = ref.turned_bound(want, met, NAMES[got.dtype])
    got = got.double().cpu().numpy()
    assert np.array_equal(got[..., rotary_dim:], want[..., rotary_dim:])
    off = ~(np.abs(got - want) <= bound)
    assert not off.any(), (int(off.sum()), np.abs(got - want)[off].max(), bound[off].min(), np.argwhere(off)[:5])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("dim, part", [(1, 0), (2, 2), (8, 8), (16, 16), (17, 16), (24, 10), (64, 64), (80, 32), (96, 48), (100, 100), (128, 128), (128, 64), (128, 8), (200, 0), (255, 254), (256, 256)])
def test_head_sizes(dtype, layout, dim, part):
    rng = np.random.default_rng(dim + part)
    positions = np.array([0, 1, 77, 4095, 131071, 2 ** 31 - 1, -1, -(2 ** 31)], np.int32)
    q, k = rows(rng, dtype, 8, 5, dim), rows(rng, dtype, 8, 2, dim)
    steps = lce.lce_rotary_steps(part)
    desc = lce.make_rotary_desc(dim, part, layout, amplitude=1.25)
    q_out, k_out = lce.lce_rotary(desc, q, k, torch.from_numpy(positions).to(DEV), steps.to(DEV))
    check(q_out, q, positions, steps, part, layout, 1.25)
    check(k_out, k, positions, steps, part, layout, 1.25)


@pytest.mark.parametrize("tokens, q_heads, k_heads", [(1, 1, 0), (1, 32, 8), (3, 13, 1), (1030, 9, 3), (777, 16, 16), (20000, 3, 1)])
def test_head_and_token_counts(tokens, q_heads, k_heads):
    rng = np.random.default_rng(tokens)
    positions = rng.integers(0, 1 << 20, tokens).astype(np.int32)
    q, k = rows(rng, BF16, tokens, q_heads, 32), rows(rng, BF16, tokens, k_heads, 32) if k_heads else None
    steps = lce.lce_rotary_steps(32)
    q_out, k_out = lce.lce_rotary(lce.make_rotary_desc(32), q, k, torch.from_numpy(positions).to(DEV), steps.to(DEV))
    check(q_out, q, positions, steps, 32, lce.ROTARY_HALVES)
    if k_heads:
        check(k_out, k, positions, steps, 32, lce.ROTARY_HALVES)
    else:
        assert k_out is None


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("layout", LAYOUTS)
@pytest.mark.parametrize("more", [0, 8, 1])  # rows on 16 bytes, and off them
def test_views_in_place_and_what_lies_between(dtype, layout, more):
    rng = np.random.default_rng(7)
    tokens, dim, part = 37, 64, 48
    wide = torch.from_numpy(rng.standard_normal((tokens, 9 * dim + more))).to(dtype).to(DEV)
    before = wide.clone()
    view = lambda t, first, heads: t.as_strided((tokens, heads, dim), (9 * dim + more, dim, 1), first * dim)
    positions = (1000 + np.arange(tokens)).astype(np.int32)
    steps = lce.lce_rotary_steps(part)
    q, k = view(wide, 0, 5), view(wide, 5, 2)
    q_out, k_out = lce.lce_rotary(lce.make_rotary_desc(dim, part, layout), q, k, torch.from_numpy(positions).to(DEV), steps.to(DEV), q, k)
    assert q_out is q and k_out is k
    check(q, view(before, 0, 5), positions, steps, part, layout)
    check(k, view(before, 5, 2), positions, steps, part, layout)
    assert torch.equal(wide[:, 7 * dim:], before[:, 7 * dim:])  # the values' part and what stands behind a row
    # heads in front of tokens
    by_head = view(before, 0, 5).transpose(0, 1).contiguous().transpose(0, 1)
    out = torch.empty_like(by_head)
    assert out.stride() == by_head.stride()
    lce.lce_rotary(lce.make_rotary_desc(dim, part, layout), by_head, None, torch.from_numpy(positions).to(DEV), steps.to(DEV), out)
    assert torch.equal(out, q)


def test_nothing_but_the_output_is_written():
    whole = torch.full((2 * 64 + 4 * 3 * 24,), 7.0, device=DEV)
    out = whole[64:64 + 4 * 3 * 24].view(4, 3, 24)
    q = torch.ones(4, 3, 24, device=DEV)
    lce.lce_rotary(lce.make_rotary_desc(24, 6), q, None, torch.arange(4, dtype=torch.int32, device=DEV), lce.lce_rotary_steps(6).to(DEV), out)
    assert bool((whole[:64] == 7).all()) and bool((whole[-64:] == 7).all()) and bool((out[..., 6:] == 1).all())


def test_turned_back_and_the_gradient():
    """Negated steps give the transposed rotation: <dy, R x> = <R' dy, x>, and R' R x = x, within the rotations' bounds."""
    rng = np.random.default_rng(11)
    tokens, heads, dim = 33, 4, 40
    x, dy = (rows(rng, F32, tokens, heads, dim) for _ in range(2))
    positions = torch.from_numpy(rng.integers(0, 1 << 17, tokens).astype(np.int32)).to(DEV)
    steps = lce.lce_rotary_steps(24, base=500.0).to(DEV)
    for layout in LAYOUTS:
        desc = lce.make_rotary_desc(dim, 24, layout)
        y, _ = lce.lce_rotary(desc, x, None, positions, steps)
        back, _ = lce.lce_rotary(desc, y, None, positions, -steps)
        dx, _ = lce.lce_rotary(desc, dy, None, positions, -steps)
        # each element twice through a rotation of (2^-23 + 2^-22 + 2^-24) of |a| + |b| <= 2 * the largest, and once more amplified by sqrt(2)
        top = max(float(x.abs().max()), float(dy.abs().max()))
        assert float((back - x).abs().max()) <= 2 * 2.0 ** -21 * 2 * top * 1.5
        a, b = (dy.double() * y.double()).sum(), (dx.double() * x.double()).sum()
        assert abs(float(a - b)) <= x.numel() * top * 2 * 2.0 ** -21 * 2 * top
        # differences along single channels: the rotation is linear, so they are exact up to the same bound
        e = torch.zeros_like(x)
        e[:, :, 5] = 1.0
        column, _ = lce.lce_rotary(desc, e, None, positions, steps)
        assert float(((dy.double() * column.double()).sum(-1) - dx[:, :, 5].double()).abs().max()) <= 4 * 2.0 ** -21 * top


def test_values_that_are_not_finite_stay_in_their_pair():
    x = torch.ones(1, 1, 32, device=DEV)
    x[0, 0, 3], x[0, 0, 20] = float("nan"), float("inf")
    y, _ = lce.lce_rotary(lce.make_rotary_desc(32), x, None, torch.tensor([5], dtype=torch.int32, device=DEV), lce.lce_rotary_steps(32).to(DEV))
    bad = (~torch.isfinite(y[0, 0])).nonzero().flatten().tolist()
    assert bad == [3, 4, 19, 20]


def test_streams_graphs_and_empty_calls():
    rng = np.random.default_rng(5)
    q = rows(rng, F16, 9, 4, 64)
    positions, steps = torch.arange(9, dtype=torch.int32, device=DEV), lce.lce_rotary_steps(64).to(DEV)
    desc = lce.make_rotary_desc(64)
    want, _ = lce.lce_rotary(desc, q, None, positions, steps)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got, _ = lce.lce_rotary(desc, q, None, positions, steps)
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    out, graph = torch.empty_like(q), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lce.lce_rotary(desc, q, None, positions, steps, out)
    positions += 3
    graph.replay()
    again, _ = lce.lce_rotary(desc, q, None, positions, steps)
    assert torch.equal(out, again) and not torch.equal(again, want)
    none, _ = lce.lce_rotary(desc, q[:0], None, positions[:0], steps)
    assert none.shape == (0, 4, 64)
