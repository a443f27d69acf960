"""Eviction against its definition: places, scores and rows are exact."""
import numpy as np
import pytest
import torch

import bounded_cache_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV

pytestmark = pytest.mark.gpu


class Pool:
    """Sequences in the cache, pages for what stays beside them, garbage everywhere else."""

    def __init__(self, lengths, budget, kv_heads=2, dim=64, page=16, seed=0, more=1):
        self.rng = rng = np.random.default_rng(seed)
        self.lengths, self.budget, self.kv_heads, self.dim, self.page = lengths, budget, kv_heads, dim, page
        counts = [-(-n // page) for n in lengths]
        kept_pages = -(-budget // page)
        pages = sum(counts) + len(lengths) * kept_pages + 3
        order = rng.permutation(pages).astype(np.int32)
        self.table = np.full((len(lengths), max(counts) + more), -1, np.int32)
        at = 0
        for b, c in enumerate(counts):
            self.table[b, :c] = order[at:at + c]
            at += c
        self.kept_table = order[at:at + len(lengths) * kept_pages].reshape(len(lengths), kept_pages)
        self.desc = lce.make_kv_desc(pages, page, kv_heads, dim)
        size = lce.lce_kv_cache_bytes(self.desc)
        self.cache = torch.from_numpy(rng.integers(0, 256, size, dtype=np.uint8)).to(DEV)  # rows of all kinds: they move as they are
        self.scores = np.exp(2 * rng.standard_normal((len(lengths), kv_heads, self.table.shape[1] * page))).astype(np.float32)

    def run(self, scores=None, table=None, **more):
        i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)
        scores = torch.from_numpy(self.scores).to(DEV) if scores is None else scores
        return lce.lce_kv_evict(self.desc, self.cache, i32(self.table if table is None else table), i32(self.lengths), scores, i32(self.kept_table), self.budget, **more)

    def rows(self, cache, slots):
        k, v = lce.lce_kv_dequantize(self.desc, cache, torch.from_numpy(np.ascontiguousarray(slots, np.int32)).to(DEV))
        return torch.cat((k, v), -1).view(torch.int32).cpu().numpy()  # bits: garbage scales may be NaN

    def check(self, first=0, recent=0, scores=None, table=None, bad=()):
        """Runs the call and compares everything.  bad: (sequence, page of its table) outside the pool."""
        before = self.cache.clone()
        given = torch.from_numpy(self.scores).to(DEV) if scores is None else scores
        kept, lengths, kept_scores = (t.cpu().numpy() for t in self.run(scores, table, first=first, recent=recent))
        have = given.cpu().numpy()
        everything = np.arange(self.desc.pages * self.page)
        want_rows = self.rows(before, everything)
        for b, n in enumerate(self.lengths):
            valid = np.ones(n, bool)
            for seq, page in bad:
                if seq == b:
                    valid[page * self.page:(page + 1) * self.page] = False
            count = min(int(valid.sum()), self.budget)
            assert lengths[b] == count
            j = np.arange(count)
            to = self.kept_table[b][j // self.page] * self.page + j % self.page
            for h in range(self.kv_heads):
                want = ref.kept(have[b, h], n, valid, self.budget, first, recent)
                assert np.array_equal(kept[b, h, :count], want) and (kept[b, h, count:] == -1).all()
                assert np.array_equal(kept_scores[b, h, :count].view(np.int32), have[b, h][want].view(np.int32)) and (kept_scores[b, h, count:] == 0).all()
                source = self.table[b][want // self.page] * self.page + want % self.page
                want_rows[to, h] = self.rows(before, source)[:, h]
        # every row of the pool: those that moved and all others as they were
        assert np.array_equal(self.rows(self.cache, everything), want_rows)
        return kept, lengths


@pytest.mark.parametrize("dim", [1, 32, 33, 64, 80, 96, 128, 160, 192, 224, 256])
@pytest.mark.parametrize("page", [16, 48])
def test_head_sizes(dim, page):
    Pool([100, 50], 37, dim=dim, page=page, seed=dim).check(first=2, recent=9)


@pytest.mark.parametrize("lengths", [[1], [0, 5], [15, 16, 17], [64, 63, 65, 0, 1], [700, 2000, 31]])
@pytest.mark.parametrize("budget", [1, 15, 16, 17, 64, 100, 2100])
def test_lengths_and_budgets(lengths, budget):
    Pool(lengths, budget, kv_heads=3, dim=32, seed=budget).check()
    Pool(lengths, budget, kv_heads=1, dim=32, seed=budget).check(first=min(4, budget), recent=budget - min(4, budget))


@pytest.mark.parametrize("length, budget, kv_heads", [(3000, 1000, 1), (9000, 4097, 2), (40000, 10000, 1), (40000, 39999, 3), (400000, 1500, 1)])
def test_long_sequences(length, budget, kv_heads):
    Pool([length], budget, kv_heads=kv_heads, dim=32, page=64, seed=length).check(first=4, recent=budget // 4)


def test_many_sequences():
    rng = np.random.default_rng(3)
    Pool([int(n) for n in rng.integers(0, 300, 150)], 40, kv_heads=4, dim=32, seed=4).check(first=1, recent=8)


@pytest.mark.parametrize("kind", ["equal", "zeros of both signs", "few values", "infinities", "nan", "all nan", "neighbours", "negative", "subnormal"])
@pytest.mark.parametrize("length", [300, 9000])
def test_scores_of_all_kinds(kind, length):
    p = Pool([length, length // 3], length // 4, dim=32, page=64, seed=5)
    rng, s = p.rng, p.scores
    if kind == "equal":
        s[:] = 0.25
    elif kind == "zeros of both signs":
        s[:] = np.where(rng.random(s.shape) < 0.5, -0.0, 0.0)
        s[:, :, 100] = 1.0
    elif kind == "few values":
        s[:] = rng.integers(0, 3, s.shape)
    elif kind == "infinities":
        s[rng.random(s.shape) < 0.4] = -np.inf
        s[rng.random(s.shape) < 0.4] = np.inf
    elif kind == "nan":
        s[rng.random(s.shape) < 0.9] = np.nan
        s[rng.random(s.shape) < 0.05] = -np.inf
    elif kind == "all nan":
        s[:] = np.nan
    elif kind == "neighbours":
        s[:] = (np.float32(1.0).view(np.int32) + rng.integers(0, 5, s.shape)).astype(np.int32).view(np.float32)
    elif kind == "negative":
        s[:] = -s
    else:
        s[:] = rng.integers(0, 1000, s.shape).astype(np.int32).view(np.float32)
    p.check(first=3, recent=10)


def test_one_choice_for_all_heads_and_strided_scores():
    p = Pool([200, 90], 33, kv_heads=3, dim=32, seed=6)
    capacity = p.table.shape[1] * p.page
    one = torch.from_numpy(p.scores[:, :1].copy()).to(DEV).expand(-1, 3, -1)
    kept, _ = p.check(scores=one)
    assert (kept == kept[:, :1]).all()
    wide = torch.zeros(2, 3, capacity + 5, device=DEV)
    wide[:, :, :capacity] = torch.from_numpy(p.scores).to(DEV)
    p.check(scores=wide)
    p.check(scores=torch.from_numpy(p.scores).to(DEV).transpose(0, 1).contiguous().transpose(0, 1))


def test_outputs_of_the_caller():
    p = Pool([100, 20], 32, dim=32, seed=7)
    want = [t.clone() for t in p.run(recent=4)]
    kept, lengths = torch.full((2, 2, 32), 9, dtype=torch.int32, device=DEV), torch.full((2,), 9, dtype=torch.int32, device=DEV)
    carried = torch.full((2, 2, 50), 7.0, device=DEV)
    got = p.run(recent=4, kept=kept, kept_lengths=lengths, kept_scores=carried)
    assert got[0] is kept and got[1] is lengths and got[2] is carried
    assert torch.equal(kept, want[0]) and torch.equal(lengths, want[1]) and torch.equal(carried[:, :, :32], want[2])
    assert bool((carried[:, :, 32:] == 7).all())


def test_pages_outside_the_pool():
    p = Pool([100, 60, 40], 64, dim=32, seed=8)
    table = p.table.copy()
    table[0, 1], table[1, 0], table[2, 2] = -1, 1 << 30, p.desc.pages
    p.check(first=4, recent=20, table=table, bad=[(0, 1), (1, 0), (2, 2)])
    # nowhere to go: places and scores are told all the same
    p.kept_table[0, 1] = -1
    before = p.cache.clone()
    kept, lengths, _ = p.run(table=table)
    assert lengths.tolist() == [64, 44, 32] and bool((kept[0] >= 0).all())
    slots = p.table[0][:6].repeat(16) * 16 + np.tile(np.arange(16), 6)
    assert np.array_equal(p.rows(p.cache, slots), p.rows(before, slots))


def test_lengths_past_the_table():
    p = Pool([64, 30], 20, dim=32, seed=9, more=0)
    p.lengths = [1000, 30]  # of the first, 64 tokens can be read; the last places are not among them
    kept, lengths, _ = (t.cpu().numpy() for t in p.run(first=2, recent=5))
    valid = np.arange(1000) < 64
    scores = np.pad(p.scores[0, 0], (0, 1000 - 64))
    assert np.array_equal(kept[0, 0], ref.kept(scores, 1000, valid, 20, 2, 5)) and lengths.tolist() == [20, 20]


def test_graph_and_side_stream():
    p = Pool([500, 300], 100, dim=64, seed=10)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)
    arguments = [p.desc, p.cache, i32(p.table), i32(p.lengths), torch.from_numpy(p.scores).to(DEV), i32(p.kept_table), 100]
    outs = dict(kept=torch.empty(2, 2, 100, dtype=torch.int32, device=DEV), kept_lengths=torch.empty(2, dtype=torch.int32, device=DEV),
                kept_scores=torch.empty(2, 2, 100, device=DEV))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lce.lce_kv_evict(*arguments, recent=10, **outs)
    for n in ([500, 300], [80, 101], [0, 100]):
        arguments[3].copy_(torch.tensor(n, dtype=torch.int32))
        graph.replay()
        got, moved = [t.clone() for t in outs.values()], p.cache.clone()
        want = lce.lce_kv_evict(*arguments, recent=10)
        assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(moved, p.cache)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lce.lce_kv_evict(*arguments, recent=10)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
