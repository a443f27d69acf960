"""Buffers that a call would write while it still reads them are refused before anything is launched; those side by side are not."""
import ctypes
from pathlib import Path

import pytest
import torch

import paper_2011_09398_b200 as lce
from paper_2011_09398_b200 import build as lce_build
from test_bounded_cache_abi import INVALID, evict_desc, rotary_desc, weights_desc

at = ctypes.c_void_p  # places that are never touched: there is no GPU, or the call is refused first


@pytest.fixture(scope="module")
def lib():
    lce_build.build()
    return lce.library()


def accepted(status):
    """Passed all checks: here, without a GPU, the launch is what fails."""
    return status not in (1, 2, 3, 6)


def evict(lib, scores, kept_scores, **change):
    d = evict_desc(**change)
    return lib.lce_kv_evict(ctypes.byref(d), at(1 << 20), at(2 << 20), at(3 << 20), at(scores), at(4 << 20), at(5 << 20), at(6 << 20), at(kept_scores) if kept_scores else None, None)


def test_scores_and_kept_scores(lib):
    # 2 sequences, 2 heads: scores of 48 in rows of 48, kept scores of 20 in rows of 20
    here = 7 << 20
    same = dict(kept_scores_seq_stride=96, kept_scores_head_stride=48)
    for there in (here, here + 4 * 96, here - 4 * 19, here + 4 * 48 - 4 * 19):
        assert evict(lib, here, there) == INVALID, there
        assert evict(lib, here, there, **same) == INVALID, there
    one_row = dict(batch=1, cache=(8, 16, 1, 64))
    assert evict(lib, here, here, **one_row) == INVALID
    assert evict(lib, here, here, scores_head_stride=0) == INVALID  # one row of scores for all heads
    # rows of kept scores apart from one another
    other = 8 << 20
    for bad in (dict(kept_scores_head_stride=0), dict(kept_scores_head_stride=19), dict(kept_scores_seq_stride=0), dict(kept_scores_seq_stride=39), dict(kept_scores_seq_stride=20, kept_scores_head_stride=20)):
        assert evict(lib, here, other, **bad) == INVALID, bad


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are accepted would be launched")
def test_scores_and_kept_scores_beside_one_another(lib):
    here, other = 7 << 20, 8 << 20
    for good in (dict(), dict(scores_head_stride=0), dict(kept_scores_seq_stride=20, kept_scores_head_stride=40), dict(batch=1, kept_scores_seq_stride=0),
                 dict(cache=(8, 16, 1, 64), kept_scores_head_stride=0)):
        assert accepted(evict(lib, here, other, **good)), good
    assert accepted(evict(lib, here, None))
    # in the same rows, behind the scores
    assert accepted(evict(lib, here, here + 4 * 48, scores_seq_stride=136, scores_head_stride=68, kept_scores_seq_stride=136, kept_scores_head_stride=68))
    assert accepted(evict(lib, here, here + 4 * 192)) and accepted(evict(lib, here + 4 * 80, here))


def test_kept_lengths_are_written_by_no_kernel_that_reads_the_lengths():
    """They may be the same memory: blocks of the kernel that chooses can begin after others of it are done."""
    text = (Path(lce.__file__).parent / "csrc" / "kv_evict.cu").read_text()
    kernels = text.split("__global__")[1:]
    kernels[-1] = kernels[-1][:kernels[-1].index("\nlce_status ")]
    reads, writes = (["kv_evict_select" in k.split("{")[0] for k in kernels if what in k] for what in ("p.lengths", "p.kept_lengths"))
    assert reads == [True] and writes == [False]


def weigh(lib, previous, out, **change):
    d = weights_desc(**change)
    return lib.lce_kv_attention_weights(ctypes.byref(d), at(1 << 20), at(2 << 20), at(3 << 20), at(4 << 20), None, at(previous) if previous else None, at(out), at(5 << 20), 1 << 40, None)


def test_previous_weights_and_out(lib):
    # 2 sequences, 2 heads, rows of 48
    here, other = 7 << 20, 8 << 20
    for there in (here + 4 * 48, here - 4 * 96):
        assert weigh(lib, there, here) == INVALID, there
    for bad in (dict(previous_head_stride=0), dict(previous_seq_stride=192), dict(out_seq_stride=48, out_head_stride=96)):
        assert weigh(lib, here, here, **bad) == INVALID, bad
    assert weigh(lib, here + 4 * 48, here, previous_head_stride=0) == INVALID  # one row for all heads, where one of them writes
    for bad in (dict(out_head_stride=0), dict(out_seq_stride=0), dict(out_seq_stride=48)):
        assert weigh(lib, None, other, **bad) == INVALID, bad


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are accepted would be launched")
def test_previous_weights_and_out_beside_one_another(lib):
    here, other = 7 << 20, 8 << 20
    assert accepted(weigh(lib, None, here)) and accepted(weigh(lib, here, here)) and accepted(weigh(lib, other, here))
    assert accepted(weigh(lib, other, here, previous_head_stride=0)) and accepted(weigh(lib, other, here, previous_head_stride=0, previous_seq_stride=0))
    assert accepted(weigh(lib, here + 4 * 48, here, decay=0.0))  # not read
    # by turns in one buffer, and strides that lead nowhere
    assert accepted(weigh(lib, here + 4 * 48, here, previous_seq_stride=192, previous_head_stride=96, out_seq_stride=192, out_head_stride=96))
    one = dict(batch=1, tokens=1, cache=(8, 16, 1, 64))
    assert accepted(weigh(lib, here, here, out_seq_stride=0, out_head_stride=0, **one)) and accepted(weigh(lib, None, here, out_seq_stride=0, out_head_stride=0, **one))


def turn(lib, q, k, q_out, k_out, **change):
    d = rotary_desc(**change)
    return lib.lce_rotary(ctypes.byref(d), at(q), at(k) if k else None, at(1 << 20), at(2 << 20), at(q_out), at(k_out) if k_out else None, None)


# queries and keys beside one another in rows of one buffer, as a projection writes them: 4 and 2 heads of 64, 3 tokens
SIDE_BY_SIDE = dict(q_token_stride=384, k_token_stride=384, q_out_token_stride=384, k_out_token_stride=384)
BUFFER, SIZE = 7 << 20, 4 * 384 * 3


def test_rotary_over_other_rows(lib):
    q, k, other = BUFFER, BUFFER + 4 * 256, BUFFER + SIZE
    for q_out, k_out in ((k, k), (q, q), (k, q), (q + 4 * 64, k), (q, k - 4 * 64), (other, other), (other, other + 4 * 255), (q, k + 4 * 384), (q + 32, k), (other, q)):
        assert turn(lib, q, k, q_out, k_out, **SIDE_BY_SIDE) == INVALID, (q_out, k_out)
    # in place, but with other strides
    for bad in (dict(q_out_token_stride=256), dict(q_out_head_stride=128), dict(k_out_token_stride=768)):
        assert turn(lib, q, k, q, k, **{**SIDE_BY_SIDE, **bad}) == INVALID, bad
    assert turn(lib, q, None, q, None, tokens=1, k_heads=0, q_out_head_stride=65) == INVALID
    # rows of an output that meet
    for bad in (dict(q_out_head_stride=0), dict(q_out_head_stride=63), dict(q_out_token_stride=0), dict(k_out_token_stride=64), dict(k_out_head_stride=0)):
        assert turn(lib, q, k, other, other + SIZE, **{**SIDE_BY_SIDE, **bad}) == INVALID, bad
    assert turn(lib, q, k, q, k, **{**SIDE_BY_SIDE, "k_head_stride": 0, "k_out_head_stride": 0}) == INVALID  # one row of k for all heads, in place


@pytest.mark.skipif(torch.cuda.is_available(), reason="calls that are accepted would be launched")
def test_rotary_beside_other_rows(lib):
    q, k, other = BUFFER, BUFFER + 4 * 256, BUFFER + SIZE
    for q_out, k_out in ((q, k), (other, k), (q, other), (other, other + 4 * 256), (other + 4 * 128, other)):
        assert accepted(turn(lib, q, k, q_out, k_out, **SIDE_BY_SIDE)), (q_out, k_out)
    assert accepted(turn(lib, q, None, q, None, k_heads=0)) and accepted(turn(lib, q, None, q, None, tokens=1, k_heads=0, q_out_token_stride=7))
    assert accepted(turn(lib, q, k, other, other + SIZE, q_token_stride=0, q_head_stride=0, k_head_stride=0))  # one row read again and again
    assert accepted(turn(lib, q, k, other, other + SIZE, q_out_token_stride=64, q_out_head_stride=192, k_out_token_stride=64, k_out_head_stride=192))  # heads in front of tokens
