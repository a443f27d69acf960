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
