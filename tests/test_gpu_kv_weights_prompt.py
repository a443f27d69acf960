"""Attention weights of many rows, 16-bit and up to 128 channels: their own kernels, in units of 256 columns or tokens and a few steps of 128 of
the other."""
import numpy as np
import pytest
import torch

import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import BF16, F16, Setup
from test_gpu_kv_weights import MARK, check, expected, run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("dim", [1, 8, 31, 32, 33, 64, 72, 96, 100, 120, 127, 128])
def test_head_sizes(dtype, dim):
    s = Setup(dtype, [300, 129], [70, 129], 2, 2, dim, seed=dim)
    check(run(s), expected(s))


@pytest.mark.parametrize("length", [1, 16, 127, 128, 129, 255, 256, 257, 513, 1500])
@pytest.mark.parametrize("rows, group", [(40, 1), (127, 1), (128, 1), (129, 1), (64, 4), (65, 4), (150, 7)])
def test_lengths_and_columns(length, rows, group):
    s = Setup(BF16, [length], [min(rows, length)], 1, group, 32, seed=length + rows)
    check(run(s), expected(s))
    if length >= rows:
        check(run(s, causal=False), expected(s, causal=False))


@pytest.mark.parametrize("window", [0, 1, 17, 128, 300, 5000])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("page", [16, 48, 128])
def test_masks(window, causal, page):
    s = Setup(F16, [700, 140, 260], [300, 140, 2], 2, 3, 64, page=page, seed=window)
    check(run(s, window=window, causal=causal), expected(s, window=window, causal=causal))


def test_batches_of_all_kinds():
    lengths = [500, 0, 1, 300, 33, 1000, 256, 70, 64, 512] * 4
    news = [500, 0, 1, 0, 33, 100, 256, 5, 64, 1] * 4
    s = Setup(BF16, lengths, news, 3, 4, 64, seed=1)
    previous = torch.rand(len(lengths), 3, s.table.shape[1] * s.page, device=DEV)
    check(run(s, previous=previous, decay=0.5), expected(s, previous=previous, decay=0.5))


@pytest.mark.parametrize("length, rows, kv_heads, group", [(6000, 400, 2, 4), (3000, 1500, 1, 8), (20000, 64, 1, 4), (2500, 600, 8, 2)])
def test_many_units(length, rows, kv_heads, group):
    s = Setup(F16, [length, length // 3], [rows, rows // 3], kv_heads, group, 64, page=64, seed=length)
    out = run(s)
    check(out, expected(s))
    assert torch.equal(out, run(s))


def test_rows_at_positions_before_the_first():
    s = Setup(BF16, [50, 300], [200, 10], 1, 2, 64, seed=2)  # 150 rows see nothing
    check(run(s), expected(s))
    check(run(s, causal=False, window=100), expected(s, causal=False, window=100))


def test_pages_outside_the_pool_and_a_short_table():
    s = Setup(BF16, [400, 300], [90, 100], 2, 2, 64, seed=3)
    table = s.table.copy()
    table[0, 2:10], table[1, 0], table[1, 18] = -1, 1 << 30, s.desc.pages
    arguments = s.arguments()
    arguments[3] = torch.from_numpy(table).to(DEV)
    out = torch.full((2, 2, s.table.shape[1] * s.page), MARK, device=DEV)
    check(lce.lce_kv_attention_weights(*arguments, out=out), expected(s, bad_tokens=[(0, slice(32, 160)), (1, slice(0, 16)), (1, slice(288, 300))]))
    arguments[3] = torch.from_numpy(np.ascontiguousarray(s.table[:, :13])).to(DEV)
    out = torch.full((2, 2, 208), MARK, device=DEV)
    want, bound = expected(s, bad_tokens=[(0, slice(208, 400)), (1, slice(208, 300))])
    check(lce.lce_kv_attention_weights(*arguments, out=out), (want[:, :, :208], bound[:, :, :208]))


def test_rows_and_keys_that_are_not_finite():
    s = Setup(F16, [400, 300], [150, 140], 1, 2, 64, seed=4)
    s.q[3, 1, 7] = float("nan")     # sees tokens up to 253
    s.q[150 + 100, 0, 0] = float("-inf")  # of the second sequence: up to 260
    out = run(s).cpu().numpy()
    assert np.isnan(out[0, 0, :254]).all() and np.isfinite(out[0, 0, 254:]).all()
    assert np.isnan(out[1, 0, :261]).all() and np.isfinite(out[1, 0, 261:]).all()
    s.q[3, 1, 7] = s.q[250, 0, 0] = 0.0
    s.k[399, 0, 3] = float("nan")  # the first sequence's last token, which its last row alone sees
    s.store()
    out = run(s).cpu().numpy()
    assert np.isnan(out[0, 0, :400]).all() and np.isfinite(out[1]).all()


@pytest.mark.parametrize("scale", [0.0, -0.3, 30.0, 1e-30])
def test_scales(scale):
    s = Setup(F16, [300], [90], 1, 2, 64, seed=5)
    check(run(s, scale=scale), expected(s, scale=scale))


def test_sizes_of_all_magnitudes():
    """Keys whose scales differ by 2^20 from token to token, rows whose sizes do from row to row."""
    s = Setup(BF16, [400], [130], 1, 2, 64, seed=6)
    rng = np.random.default_rng(0)
    s.k *= torch.from_numpy(2.0 ** rng.integers(-20, 1, (400, 1, 1))).to(BF16).to(DEV)
    s.q *= torch.from_numpy(2.0 ** rng.integers(-30, 3, (130, 1, 1))).to(BF16).to(DEV)
    s.store()
    check(run(s), expected(s))


def test_graph_of_growing_sequences_and_one_workspace():
    s = Setup(BF16, [700, 500], [200, 100], 2, 2, 64, seed=7)
    arguments = s.arguments()
    room = torch.empty(lce.lce_kv_attention_weights_workspace_bytes(s.desc, 2, 300, 4, s.table.shape[1], BF16), dtype=torch.uint8, device=DEV)
    out = torch.full((2, 2, s.table.shape[1] * s.page), MARK, device=DEV)
    lengths = arguments[4]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lce.lce_kv_attention_weights(*arguments, out=out, workspace=room)
    for grown in ([200, 100], [333, 0], [700, 500]):
        lengths.copy_(torch.tensor(grown, dtype=torch.int32))
        out.fill_(MARK)
        room.fill_(0xFF)
        graph.replay()
        want = torch.full_like(out, MARK)
        lce.lce_kv_attention_weights(*arguments, out=want)
        assert torch.equal(out, want)
    check(out, expected(s))
    assert lce.lce_device_status() == 0


def test_many_rows_after_an_expired_wait():
    s = Setup(BF16, [300], [100], 1, 2, 64, seed=8)
    lce.lce_device_wait_probe(20_000)
    torch.cuda.synchronize()
    try:
        with pytest.raises(lce.LceError) as e:
            run(s)
        assert e.value.status == 5
    finally:
        lce.lce_device_status_reset()
    check(run(s), expected(s))


@pytest.mark.parametrize("rows", [1, 90])
@pytest.mark.parametrize("causal", [True, False])
def test_the_widest_window(rows, causal):
    s = Setup(F16, [300], [rows], 1, 2, 64, seed=9)
    check(run(s, window=2 ** 31 - 1, causal=causal), expected(s, causal=causal))
