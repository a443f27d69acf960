"""Attention weights by token against the definition in 64 bits; bounded_cache_reference.weights derives the bounds."""
import numpy as np
import pytest
import torch

import bounded_cache_reference as ref
import kv_reference
import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import BF16, F16, F32, Setup

pytestmark = pytest.mark.gpu
MARK = 12345.0


def expected(s, scale=None, causal=True, window=0, previous=None, decay=1.0, bad_tokens=()):
    """[sequences, kv heads, tokens of the table] and bounds; MARK behind each sequence."""
    scale = s.dim ** -0.5 if scale is None else scale
    k, ks = kv_reference.quantized(s.k.double().cpu().numpy())
    q = s.q.double().cpu().numpy()
    capacity = s.table.shape[1] * s.page
    out, bound = np.full((len(s.lengths), s.kv_heads, capacity), MARK), np.zeros((len(s.lengths), s.kv_heads, capacity))
    row = token = 0
    for b, (n, new) in enumerate(zip(s.lengths, s.news)):
        t, p = np.arange(n), n - new + np.arange(new)[:, None]
        shown = np.ones((new, n), bool)
        if causal:
            shown &= t <= p
        if window:
            shown &= t > p - window
        for which, bad in bad_tokens:
            if which == b:
                shown[:, bad] = False
        out[b, :, :n], bound[b, :, :n] = ref.weights(q[row:row + new], k[token:token + n], ks[token:token + n], shown, scale)
        if previous is not None and decay:
            old = max(n - new, 0)
            carried = float(np.float32(decay)) * previous[b, :, :old].double().cpu().numpy()
            out[b, :, :old] += carried
            bound[b, :, :old] += 2.0 ** -24 * np.abs(out[b, :, :old])
        row, token = row + new, token + n
    return out, bound


def run(s, previous=None, **more):
    capacity = s.table.shape[1] * s.page
    out = torch.full((len(s.lengths), s.kv_heads, capacity), MARK, device=DEV)
    return lce.lce_kv_attention_weights(*s.arguments(), previous=previous, out=out, **more)


def check(got, want):
    out, bound = want
    got = got.double().cpu().numpy()
    with np.errstate(invalid="ignore"):
        off = ~(np.abs(got - out) <= bound) & ~(np.isnan(got) & np.isnan(out))
    assert not off.any(), (int(off.sum()), np.abs(got - out)[off].max(), bound[off].min(), np.argwhere(off)[:5])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [1, 8, 17, 32, 40, 64, 80, 96, 100, 128, 160, 192, 224, 255, 256])
def test_head_sizes(dtype, dim):
    s = Setup(dtype, [70, 1, 33], [1, 1, 1], 2, 4, dim, seed=1)
    check(run(s), expected(s))
    s = Setup(dtype, [50, 21], [5, 3], 1, 3, dim, seed=2)
    check(run(s), expected(s))
    s = Setup(dtype, [150], [40], 1, 2, dim, seed=3)
    check(run(s), expected(s))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("group", [1, 2, 3, 5, 7, 8, 9, 15, 16, 17, 40])
def test_groups_and_rows(dtype, group):
    s = Setup(dtype, [130, 16, 77], [1, 1, 1], 2, group, 64, seed=group)
    check(run(s), expected(s))
    s = Setup(dtype, [90, 0, 31, 2], [3, 0, 31, 2], 1, group, 32, seed=group)
    check(run(s), expected(s))


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("window", [0, 1, 15, 16, 17, 100, 5000])
@pytest.mark.parametrize("news", [[1, 1, 1], [7, 1, 3], [200, 40, 0]])
def test_masks(causal, window, news):
    s = Setup(BF16, [400, 40, 129], news, 2, 2, 64, seed=4)
    check(run(s, causal=causal, window=window), expected(s, causal=causal, window=window))


@pytest.mark.parametrize("page", [16, 48, 128])
@pytest.mark.parametrize("length", [1, 15, 16, 17, 127, 128, 129, 1000, 5000])
def test_lengths_and_pages(page, length):
    s = Setup(F16, [length], [1], 3, 4, 64, page=page, seed=length)
    check(run(s), expected(s))


def test_long_sequences_beside_short_ones():
    s = Setup(BF16, [20000, 3, 700, 0, 9000], [1, 1, 1, 0, 1], 2, 4, 64, page=64, seed=8)
    check(run(s), expected(s))
    s = Setup(F32, [9000, 3, 700], [2, 3, 30], 1, 4, 64, page=64, seed=9)
    check(run(s), expected(s))


@pytest.mark.parametrize("decay", [1.0, 0.75, 0.0, -0.5])
@pytest.mark.parametrize("in_place", [False, True])
def test_previous_weights(decay, in_place):
    s = Setup(F16, [300, 17, 64], [1, 5, 64], 2, 2, 64, seed=5)
    rng = np.random.default_rng(1)
    previous = torch.from_numpy(rng.random((3, 2, s.table.shape[1] * s.page)).astype(np.float32)).to(DEV)
    for b, n in enumerate(s.lengths):
        previous[b, :, n - s.news[b]:] = float("nan") if not in_place else MARK  # what new tokens have there does not count
    want = expected(s, previous=previous, decay=decay)
    if not in_place:
        if decay == 0.0:
            previous.fill_(float("nan"))  # not read
        check(run(s, previous=previous, decay=decay), want)
    else:
        got = lce.lce_kv_attention_weights(*s.arguments(), previous=previous, out=previous, decay=decay)
        assert got is previous
        check(got, want)


def test_strided_buffers():
    s = Setup(BF16, [90, 33], [1, 1], 2, 3, 64, seed=6)
    capacity = s.table.shape[1] * s.page
    want = expected(s)
    wide = torch.full((2, 2, capacity + 7), MARK, device=DEV)
    lce.lce_kv_attention_weights(*s.arguments(), out=wide)
    check(wide[:, :, :capacity], want)
    assert bool((wide[:, :, capacity:] == MARK).all())
    by_head = torch.full((2, 2, capacity), MARK, device=DEV).transpose(0, 1)
    lce.lce_kv_attention_weights(*s.arguments(), out=by_head)
    check(by_head, want)
    # q as a view of a wider projection, off its 16 bytes
    wide_q = torch.zeros(2, 6 * 64 + 3, dtype=BF16, device=DEV)
    view = wide_q.as_strided((2, 6, 64), (6 * 64 + 3, 64, 1), 1)
    view.copy_(s.q)
    arguments = s.arguments()
    arguments[1] = view
    out = torch.full((2, 2, capacity), MARK, device=DEV)
    check(lce.lce_kv_attention_weights(*arguments, out=out), want)


def test_sequences_without_rows_or_tokens():
    s = Setup(F32, [64, 0, 40], [0, 0, 0], 2, 2, 32, seed=7)
    previous = torch.ones(3, 2, s.table.shape[1] * s.page, device=DEV)
    out = run(s, previous=previous, decay=0.5)
    assert bool((out[0, :, :64] == 0.5).all()) and bool((out[2, :, :40] == 0.5).all())
    assert bool((out[0, :, 64:] == MARK).all()) and bool((out[1] == MARK).all()) and bool((out[2, :, 40:] == MARK).all())
    # more rows than tokens: those at negative positions see nothing
    s = Setup(F32, [3, 20], [5, 1], 1, 2, 32, seed=7)
    check(run(s), expected(s))


@pytest.mark.parametrize("news", [[1, 1], [20, 3]])
def test_pages_outside_the_pool_and_a_short_table(news):
    s = Setup(BF16, [100, 70], news, 2, 2, 64, seed=10)
    table = s.table.copy()
    table[0, 2], table[1, 0] = -1, 1 << 30
    arguments = s.arguments()
    arguments[3] = torch.from_numpy(table).to(DEV)
    bad = [(0, slice(32, 48)), (1, slice(0, 16))]
    out = torch.full((2, 2, s.table.shape[1] * s.page), MARK, device=DEV)
    check(lce.lce_kv_attention_weights(*arguments, out=out), expected(s, bad_tokens=bad))
    # positions follow from the length, also where the table is shorter
    arguments[3] = torch.from_numpy(np.ascontiguousarray(s.table[:, :4])).to(DEV)
    out = torch.full((2, 2, 64), MARK, device=DEV)
    want, bound = expected(s, bad_tokens=[(0, slice(64, 100)), (1, slice(64, 70))])
    check(lce.lce_kv_attention_weights(*arguments, out=out), (want[:, :, :64], bound[:, :, :64]))


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("news", [[1, 1], [33, 40]])
def test_rows_and_keys_that_are_not_finite(dtype, news):
    s = Setup(dtype, [90, 50], news, 1, 2, 64, seed=11)
    s.q[0, 0, 5] = float("inf")
    first_hi = s.lengths[0] - news[0] + 1
    out = run(s).cpu().numpy()
    assert np.isnan(out[0, 0, :first_hi]).all() and np.isfinite(out[0, 0, first_hi:]).all() and np.isfinite(out[1]).all()
    s.q[0, 0, 5] = 0.0
    s.k[s.lengths[0] + 49, 0, 3] = float("nan")  # the second sequence's last token: only its last row sees it
    s.store()
    out = run(s).cpu().numpy()
    assert np.isfinite(out[0]).all() and np.isnan(out[1, 0, :50]).all()
    # masked: nobody sees it
    out = lce.lce_kv_attention_weights(s.desc, s.q, s.cache, s.arguments()[3], torch.tensor([90, 49], dtype=torch.int32, device=DEV), s.arguments()[5],
                                       out=torch.full((2, 1, s.table.shape[1] * s.page), MARK, device=DEV))
    assert bool(torch.isfinite(out).all())


@pytest.mark.parametrize("scale", [0.0, -0.3, 30.0, 1e-30])
def test_scales(scale):
    s = Setup(F16, [80, 33], [2, 1], 1, 4, 64, seed=12)
    check(run(s, scale=scale), expected(s, scale=scale))


def test_sums_are_the_rows():
    """Every row's weights add up to one, whatever form the call takes; and the same bits come again."""
    for dtype, lengths, news, group in ((BF16, [3000, 100], [1, 1], 4), (F16, [700], [300], 4), (F32, [500, 2], [9, 2], 3), (BF16, [2049], [1000], 8)):
        s = Setup(dtype, lengths, news, 2, group, 128, seed=13)
        out = run(s)
        assert torch.equal(out, run(s))
        for b, n in enumerate(lengths):
            total = out[b, :, :n].double().sum(-1).cpu().numpy()
            # errors of single weights as expected() bounds them at |scores| < 40: 2^-14 at most
            assert (np.abs(total - news[b] * group) <= 2.0 ** -14 * news[b] * group).all()


def test_graph_of_growing_sequences_and_workspaces():
    s = Setup(BF16, [200, 90], [1, 1], 2, 4, 64, seed=14)
    arguments = s.arguments()
    bytes_ = lce.lce_kv_attention_weights_workspace_bytes(s.desc, 2, 2, 8, s.table.shape[1], BF16)
    room = torch.empty(bytes_, dtype=torch.uint8, device=DEV)
    out = torch.full((2, 2, s.table.shape[1] * s.page), MARK, device=DEV)
    lengths = torch.tensor([150, 40], dtype=torch.int32, device=DEV)
    arguments[4] = lengths
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lce.lce_kv_attention_weights(*arguments, out=out, workspace=room)
    for grown in ([151, 41], [200, 90], [1, 0]):
        lengths.copy_(torch.tensor(grown, dtype=torch.int32))
        out.fill_(MARK)
        room.fill_(0xFF)
        graph.replay()
        want = torch.full_like(out, MARK)
        lce.lce_kv_attention_weights(*arguments, out=want)
        assert torch.equal(out, want)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = lce.lce_kv_attention_weights(*arguments, out=torch.full_like(out, MARK))
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("dim, group, news", [(64, 3, [1, 1]), (128, 4, [6, 2]), (192, 9, [1, 3])])
def test_tables_too_wide_for_scores_to_be_kept(dtype, dim, group, news):
    s = Setup(dtype, [300, 70], news, 1, group, dim, seed=15, table_extra=1000000)
    room = lce.lce_kv_attention_weights_workspace_bytes(s.desc, 2, sum(news), group, s.table.shape[1], dtype)
    assert room < 128 << 20  # the scores of such a table would be above 256 MB
    out = run(s, window=150)
    narrow = Setup(dtype, [300, 70], news, 1, group, dim, seed=15)
    want, bound = expected(narrow, window=150)
    n = want.shape[2]
    check(out[:, :, :n], (want, bound))
    assert bool((out[:, :, n:] == MARK).all())


@pytest.mark.parametrize("group", [129, 260])
def test_more_columns_than_are_joined_at_once(group):
    s = Setup(F32, [70, 33], [1, 2], 1, group, 32, seed=16)
    check(run(s), expected(s))
