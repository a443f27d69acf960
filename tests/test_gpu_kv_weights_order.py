"""Attention weights by token of calls without rows of q, whose lengths the kernel in front has just written: here a binary convolution, which
lets the next kernel take its place before its own outputs are there."""
import numpy as np
import pytest
import torch

import oracle
import paper_2011_09398_b200 as lce
from gpu_util import DEV, to_dev_words
from test_gpu_kv_attention import F32, Setup

pytestmark = pytest.mark.gpu
OUTPUTS = 40


@pytest.mark.parametrize("channels, positions", [(64, 8), (1024, 56)])
def test_lengths_written_right_before_a_call_without_rows(channels, positions):
    rng = np.random.default_rng(channels)
    s = Setup(F32, [64, 48, 30, 0], [0, 0, 0, 0], 2, 2, 32, seed=1, table_extra=1)
    batch, capacity = 4, s.table.shape[1] * s.page
    a = (2 * rng.integers(0, 2, size=(1, positions, positions, channels)) - 1).astype(np.int8)
    desc = lce.make_desc(1, positions, positions, channels, OUTPUTS, kernel=(1, 1), out_type=lce.OUT_INT32, kernel_choice=lce.KERNEL_TENSOR, weights_packed=1)
    images, sums = [], []
    for _ in range(4):
        w = (2 * rng.integers(0, 2, size=(OUTPUTS, 1, 1, channels)) - 1).astype(np.int8)
        images.append(lce.lce_bconv2d_pack_weights(desc, to_dev_words(oracle.bitpack_pm1(w))))
        sums.append(oracle.bconv2d_acc(a, w).reshape(-1, OUTPUTS)[-1, :batch])  # the last position's first ones: the lengths
    bits = to_dev_words(oracle.bitpack_pm1(a))
    acc = torch.empty((1, positions, positions, OUTPUTS), dtype=torch.int32, device=DEV)
    lengths = acc.view(-1, OUTPUTS)[-1, :batch]
    previous = torch.from_numpy(rng.random((batch, 2, capacity)).astype(np.float32)).to(DEV)
    q, starts, table = s.arguments()[1], s.arguments()[5], s.arguments()[3]
    outs = []

    def run():
        outs.clear()
        for image in images:
            lce.lce_bconv2d(desc, bits, image, out=acc)
            outs.append(lce.lce_kv_attention_weights(s.desc, q, s.cache, table, lengths, starts, previous=previous, decay=0.5, out=torch.full_like(previous, -1.0)))

    def check():
        for out, n in zip(outs, sums):
            there = torch.arange(capacity, device=DEV) < torch.from_numpy(n.astype(np.int64)).to(DEV).clamp(0, capacity)[:, None, None]
            assert torch.equal(out, torch.where(there, 0.5 * previous, -1.0))
    for _ in range(3):
        run()
        check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        graph.replay()
        check()
