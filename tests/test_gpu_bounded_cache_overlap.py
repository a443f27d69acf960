"""Buffers of the bounded cache's calls that share memory: refused where a call would write what it still reads, taken where they lie side by side."""
import numpy as np
import pytest
import torch

import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import Setup
from test_gpu_kv_evict import Pool

pytestmark = pytest.mark.gpu


def test_scores_and_kept_scores_of_one_buffer():
    p = Pool([200, 90], 33, kv_heads=3, dim=32, seed=1)
    capacity = p.table.shape[1] * p.page
    want = [t.clone() for t in p.run(recent=4)]
    buffer = torch.zeros(2, 3, capacity + 33, device=DEV)
    scores = buffer[:, :, :capacity]
    scores.copy_(torch.from_numpy(p.scores))
    before, cache = buffer.clone(), p.cache.clone()
    for kept_scores in (scores, buffer, buffer[:, :, 5:], buffer[:, :, capacity - 1:]):
        with pytest.raises(ValueError, match="kept_scores must not be memory of scores"):
            p.run(scores, recent=4, kept_scores=kept_scores)
    one = scores[:, :1].expand(-1, 3, -1)
    with pytest.raises(ValueError, match="kept_scores must not be memory of scores"):
        p.run(one, recent=4, kept_scores=scores)
    for kept_scores in (torch.zeros(2, 1, 33, device=DEV).expand(-1, 3, -1), torch.zeros(1, 3, 33, device=DEV).expand(2, -1, -1), torch.zeros(200, device=DEV).as_strided((2, 3, 33), (90, 30, 1))):
        with pytest.raises(ValueError, match="apart"):
            p.run(scores, recent=4, kept_scores=kept_scores)
    assert torch.equal(buffer, before) and torch.equal(p.cache, cache)
    got = p.run(scores, recent=4, kept_scores=buffer[:, :, capacity:])
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(scores, before[:, :, :capacity])


def test_sums_carried_in_two_buffers_in_turn():
    p = Pool([300, 120], 64, kv_heads=2, dim=32, seed=2)
    capacity = p.table.shape[1] * p.page
    turns = [torch.from_numpy(p.scores).to(DEV), torch.full((2, 2, capacity), 9.0, device=DEV)]
    want = [t.clone() for t in p.run(first=2, recent=8)]
    kept, lengths, kept_scores = p.run(turns[0], first=2, recent=8, kept_scores=turns[1])
    assert kept_scores is turns[1] and torch.equal(kept, want[0]) and torch.equal(lengths, want[1]) and torch.equal(turns[1][:, :, :64], want[2])
    assert bool((turns[1][:, :, 64:] == 9).all())


@pytest.mark.parametrize("sequences, kv_heads, length, budget", [(1, 1, 100, 40), (3, 4, 500, 40), (90, 16, 200, 40), (4, 8, 40000, 1000)])
def test_lengths_in_place(sequences, kv_heads, length, budget):
    """More blocks than the GPU takes at once: those of a sequence's later heads begin when the first head's are done."""
    lengths = [0, length, budget, budget - 1, 1][:sequences] + [length - 7 * i % 97 for i in range(max(sequences - 5, 0))]
    lengths[-1] = length
    p = Pool(lengths, budget, kv_heads=kv_heads, dim=32, page=64 if length > 1000 else 16, seed=sequences)
    want = [t.clone() for t in p.run(first=3, recent=9)]
    cache = p.cache.clone()
    assert want[1].tolist() == [min(n, budget) for n in lengths]
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)
    carried, scores = i32(p.lengths), torch.from_numpy(p.scores).to(DEV)
    for start in (lengths, lengths[::-1][:sequences]):
        carried.copy_(torch.tensor(start, dtype=torch.int32))
        same = torch.equal(carried.cpu(), torch.tensor(lengths, dtype=torch.int32))
        wanted = want if same else [t.clone() for t in lce.lce_kv_evict(p.desc, p.cache, i32(p.table), carried.clone(), scores, i32(p.kept_table), budget, first=3, recent=9)]
        got = lce.lce_kv_evict(p.desc, p.cache, i32(p.table), carried, scores, i32(p.kept_table), budget, first=3, recent=9, kept_lengths=carried)
        assert got[1] is carried and all(torch.equal(a, b) for a, b in zip(got, wanted))
        if same:
            assert torch.equal(p.cache, cache)


@pytest.mark.parametrize("dtype, lengths, news", [(torch.float32, [100, 60], [1, 1]), (torch.bfloat16, [400, 300], [150, 140])])
def test_previous_weights_and_out_of_one_buffer(dtype, lengths, news):
    s = Setup(dtype, lengths, news, 2, 2, 64, seed=3)
    capacity = s.table.shape[1] * s.page
    start = torch.rand(2, 2, capacity, device=DEV)
    call = lambda previous, out, **more: lce.lce_kv_attention_weights(*s.arguments(), previous=previous, out=out, decay=0.5, **more)
    want = call(start, torch.zeros_like(start))
    # rows by turns: the sums before and the new ones
    buffer = torch.zeros(2, 2, 2, capacity + 1, device=DEV)
    buffer[:, :, 0, :capacity] = start
    old, new = buffer[:, :, 0], buffer[:, :, 1]
    before = buffer.clone()
    for previous, out in ((old, old[:, :, 1:]), (old[:, :, 1:], old), (old, buffer[:, 0]), (old[:, :1].expand(-1, 2, -1), old), (old, buffer.view(-1).as_strided(old.shape, (2 * capacity + 2, capacity + 1, 1)))):
        with pytest.raises(ValueError, match="previous"):
            call(previous, out)
    for out in (torch.zeros(2, 1, capacity, device=DEV).expand(-1, 2, -1), torch.zeros(4 * capacity, device=DEV).as_strided(start.shape, (capacity, capacity - 1, 1))):
        with pytest.raises(ValueError, match="apart"):
            call(None, out)
    assert torch.equal(buffer, before)
    assert call(old, new) is new and torch.equal(new[:, :, :capacity], want) and torch.equal(old, before[:, :, 0])
    # one row of sums for all heads, as it is read
    one = old[:, :1].expand(-1, 2, -1)
    assert torch.equal(call(one, torch.zeros_like(start)), call(one.contiguous(), torch.zeros_like(start)))
    assert call(old, old) is old and torch.equal(old[:, :, :capacity], torch.where(want == 0, before[:, :, 0, :capacity], want))


@pytest.mark.parametrize("tokens", [1, 5])
def test_rotary_over_other_rows(tokens):
    wide = torch.rand(tokens, 8 * 64, device=DEV)
    before = wide.clone()
    view = lambda first, heads: wide.as_strided((tokens, heads, 64), (8 * 64, 64, 1), 64 * first)
    q, k = view(0, 4), view(4, 2)
    desc, positions, steps = lce.make_rotary_desc(64), torch.arange(tokens, dtype=torch.int32, device=DEV) + 3, lce.lce_rotary_steps(64).to(DEV)
    call = lambda **outs: lce.lce_rotary(desc, q, k, positions, steps, **outs)
    for outs in (dict(q_out=view(2, 4)), dict(q_out=view(4, 4)), dict(k_out=view(0, 2)), dict(q_out=q, k_out=view(3, 2)), dict(q_out=torch.empty(tokens, 1, 64, device=DEV).expand(-1, 4, -1))):
        with pytest.raises(lce.LceError) as e:
            call(**outs)
        assert e.value.status == 1
    with pytest.raises(ValueError, match="strides"):
        call(q_out=wide.as_strided((tokens, 4, 64), (8 * 64, 128, 1)))
    assert torch.equal(wide, before)
    want = call()
    # keys to where the values were, queries in place
    got = call(q_out=q, k_out=view(6, 2))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(k, before.as_strided(k.shape, k.stride(), 64 * 4))
