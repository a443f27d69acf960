"""Attention weights of many rows beside keys and rows of q that are much larger: what the kernels work on together (128 tokens, 128 columns) shares
a power of two, and loses nothing above the limits that lce.h names."""
import pytest
import torch

from test_gpu_kv_attention import BF16, F16, Setup
from test_gpu_kv_weights import check, expected, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("power", [10, 18, 20])
@pytest.mark.parametrize("token", [100, 129, 299])
def test_a_large_key_that_rows_in_front_do_not_see(power, token):
    """They see the other tokens alone, whose scales are 2^-28 of the largest at least: the bounds are those of what they see."""
    s = Setup(BF16, [300], [250], 1, 2, 64, seed=power)  # rows at positions 50 ..
    s.k[token] *= 2.0 ** power
    s.q[token - 50:] = 0  # rows that see it: equal weights, whatever the keys
    s.store()
    largest = s.k.float().abs().view(300, 2, 32).amax(-1)
    assert float(largest.min()) * 2.0 ** 27 > float(largest.max())  # scales are a seventh of these, by up to a step of 2^-7 more
    check(run(s), expected(s))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("power", [8, 14])
def test_a_large_element_of_one_row(dtype, power):
    """In a channel that all keys have 0 in, so that the scores stay what they are; the other rows' bounds are their own."""
    s = Setup(dtype, [300], [250], 1, 2, 64, seed=power)
    s.k[:, :, 5] = 0
    s.q[30, 1, 5] = 2.0 ** power
    s.q[200, 0, 5] = -(2.0 ** power)
    s.store()
    check(run(s), expected(s))


def test_a_key_that_is_no_number_leaves_the_others_their_size():
    s = Setup(BF16, [300], [250], 1, 2, 64, seed=3)
    s.k[290, 0, 7] = float("nan")  # seen by the last ten rows alone
    s.store()
    assert bool(torch.isnan(run(s)[0, 0, :300]).all())
    # without these rows and their tokens, which are still in the cache
    s.lengths, s.news, s.q, s.k = [290], [240], s.q[:240], s.k[:290]
    check(run(s), expected(s))
