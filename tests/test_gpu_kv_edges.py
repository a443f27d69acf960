"""Attention over the 4-bit cache where its definition has edges; kv_reference.attention derives the bounds."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import BF16, F16, F32, NAMES, Setup, check

pytestmark = pytest.mark.gpu


def expected_of_lengths(s, lengths, causal, window):
    """By the definition, where the sequences are `lengths` tokens long and the table holds s.lengths of them."""
    (k, ks), (v, vs) = (ref.quantized(t.double().cpu().numpy()) for t in (s.k, s.v))
    q = s.q.double().cpu().numpy()
    out, bound = np.zeros(q.shape), np.zeros(q.shape)
    row = token = 0
    for held, n, new in zip(s.lengths, lengths, s.news):
        t = np.arange(held)
        for p in range(n - new, n):
            shown = np.ones(held, bool)
            if causal:
                shown &= t <= p
            if window:
                shown &= t > p - window
            out[row], bound[row] = ref.attention(q[row], *(a[token:token + held] for a in (k, v, ks, vs)), shown, s.dim ** -0.5, NAMES[s.dtype])
            row += 1
        token += held
    return out, bound


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 5, 40])
@pytest.mark.parametrize("held,news,page,table", [([64, 48], [1, 1], 16, 4), ([64, 64], [6, 30], 16, 4), ([1200], [300], 48, 25)])
def test_positions_where_the_table_is_shorter_than_the_sequence(dtype, causal, window, held, news, page, table):
    """Tokens behind the table are masked; the rows stand where the sequence's own length puts them."""
    s = Setup(dtype, held, news, 2, 4, 64, page=page, seed=50, table_extra=0)
    assert s.table.shape[1] == table
    for past in (3, 10, 150, 2 ** 31 - 1 - held[0]):
        lengths = [held[0] + past] + held[1:]
        args = s.arguments()
        args[4] = torch.tensor(lengths, dtype=torch.int32, device=DEV)
        check(lce.lce_kv_attention(*args, causal=causal, window=window), expected_of_lengths(s, lengths, causal, window))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [1e6, 1.0, 1e-9])
@pytest.mark.parametrize("new", [1, 12])
@pytest.mark.parametrize("at", [5, 35])
def test_values_next_to_a_block_that_is_not_finite(dtype, size, new, at):
    """A block of NaN leaves the others of its tile as they are, whatever their size."""
    s = Setup(dtype, [40], [new], 1, 2, 64, seed=51)
    s.v *= size
    s.v[at, 0, 40] = float("inf")
    s.store()
    out, bound = s.expected()
    rows = torch.arange(new) >= at - (40 - new)  # those that see it
    assert np.isfinite(out[:, :, :32]).all() and np.isnan(out[rows.numpy()][:, :, 32:]).all() and np.isfinite(out[~rows.numpy()]).all()
    check(lce.lce_kv_attention(*s.arguments()), (out, bound))


def test_many_rows_that_are_not_finite_and_see_nothing():
    """A row that sees no token is 0 whatever it holds."""
    s = Setup(F16, [700, 20], [500, 64], 2, 4, 64, page=16, seed=52, table_extra=400)
    want = s.expected()
    s.q[503, 1, 5], s.q[520] = float("inf"), float("nan")  # at positions -41 and -24
    got = lce.lce_kv_attention(*s.arguments())
    assert not got[500:544].any()
    check(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("size", [-102, -98, -90, -60, 0, 60])
def test_values_of_any_size_over_a_long_sequence(dtype, size):
    """Equal weights: the sum of 300000 of them stays within fp32 next to the smallest values."""
    tokens = 300000
    s = Setup(dtype, [tokens], [1], 1, 1, 32, page=128, seed=53, q_size=0.0)
    s.v = torch.ldexp(torch.ones(tokens, 1, 32, device=DEV), torch.tensor(size, device=DEV)).to(dtype) * 7
    s.store()
    got = lce.lce_kv_attention(*s.arguments()).double().cpu().numpy()
    # all the values are the same: weights and their sum are exact powers of two times counts, the rest is the output's rounding
    np.testing.assert_allclose(got, 7 * 2.0 ** size, rtol=2.0 ** -8 if dtype == BF16 else (tokens // 16 + 65) * 2.0 ** -23, atol=0)
