"""Attention over the 4-bit cache against the definition in 64 bits; kv_reference.attention derives the bounds."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV

pytestmark = pytest.mark.gpu
NAMES = {torch.float32: "float32", torch.float16: "float16", torch.bfloat16: "bfloat16"}
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16


class Setup:
    """Sequences of `lengths` tokens in the cache, the last `news` of them with rows of q; pages in no order, garbage behind them."""

    def __init__(self, dtype, lengths, news, kv_heads, group, dim, page=16, seed=0, q_size=1.0, spare_pages=2, table_extra=1):
        rng = np.random.default_rng(seed + 31 * dim + len(lengths))
        self.dtype, self.lengths, self.news, self.kv_heads, self.group, self.dim, self.page = dtype, lengths, news, kv_heads, group, dim, page
        counts = [-(-n // page) for n in lengths]
        pages = sum(counts) + spare_pages
        order = rng.permutation(pages)
        self.desc = lce.make_kv_desc(pages, page, kv_heads, dim)
        self.cache = torch.full((lce.lce_kv_cache_bytes(self.desc),), 0xFF, dtype=torch.uint8, device=DEV)  # NaN wherever nothing is stored
        table = np.full((len(lengths), max(counts + [0]) + table_extra), -1, np.int32)
        slots, at = [], 0
        for b, n in enumerate(lengths):
            table[b, :counts[b]] = order[at:at + counts[b]]
            at += counts[b]
            t = np.arange(n)
            slots.append(table[b][t // page] * page + t % page)
        self.table, self.slots = table, slots
        to = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(dtype).to(DEV)
        total = sum(lengths)
        stand_out = 1 + 6 * (rng.random((kv_heads, dim)) < 0.06)
        self.k, self.v = to(rng.standard_normal((total, kv_heads, dim)) * stand_out), to(rng.standard_normal((total, kv_heads, dim)) * np.exp(rng.standard_normal((total, 1, 1))))
        self.q = to(rng.standard_normal((sum(news), kv_heads * group, dim)) * q_size)
        self.store()

    def store(self):
        if sum(self.lengths):
            lce.lce_kv_quantize(self.desc, self.k, self.v, torch.from_numpy(np.concatenate(self.slots).astype(np.int32)).to(DEV), self.cache)

    def arguments(self):
        i32 = lambda a: torch.tensor(a, dtype=torch.int32, device=DEV)
        starts = np.concatenate([[0], np.cumsum(self.news)])
        return [self.desc, self.q, self.cache, i32(self.table), i32(self.lengths), i32(starts)]

    def expected(self, scale=None, causal=True, window=0, bad_tokens=()):
        scale = self.dim ** -0.5 if scale is None else scale
        (k, ks), (v, vs) = (ref.quantized(t.double().cpu().numpy()) for t in (self.k, self.v))
        q = self.q.double().cpu().numpy()
        out, bound = np.zeros(q.shape), np.zeros(q.shape)
        row = token = 0
        for b, (n, new) in enumerate(zip(self.lengths, self.news)):
            t = np.arange(n)
            for i in range(new):
                p = n - new + i
                shown = np.ones(n, bool)
                if causal:
                    shown &= t <= p
                if window:
                    shown &= t > p - window
                for s, bad in bad_tokens:
                    if s == b:
                        shown[bad] = False
                out[row], bound[row] = ref.attention(q[row], k[token:token + n], v[token:token + n], ks[token:token + n], vs[token:token + n], shown, scale, NAMES[self.dtype])
                row += 1
            token += n
        return out, bound


def check(got, want):
    out, bound = want
    got = got.double().cpu().numpy()
    assert got.shape == out.shape
    with np.errstate(invalid="ignore"):
        off = ~(np.abs(got - out) <= bound) & ~(np.isnan(got) & np.isnan(out))
    assert not off.any(), (int(off.sum()), np.abs(got - out)[off].max(), bound[off].min(), np.argwhere(off)[:5])


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [1, 8, 17, 32, 40, 64, 80, 96, 100, 128, 160, 192, 224, 255, 256])
def test_head_sizes(dtype, dim):
    s = Setup(dtype, [70, 1, 33], [1, 1, 1], 2, 4, dim, seed=1)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())
    s = Setup(dtype, [50, 21], [5, 3], 1, 3, dim, seed=2)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kv_heads,group", [(1, 1), (3, 1), (1, 2), (2, 3), (1, 7), (2, 8), (1, 9), (1, 16), (2, 24), (1, 71)])
def test_head_layouts(dtype, kv_heads, group):
    s = Setup(dtype, [45, 128], [1, 1], kv_heads, group, 64, seed=3)
    check(lce.lce_kv_attention(*s.arguments()[:5]), s.expected())
    s = Setup(dtype, [45, 130], [2, 4], kv_heads, group, 64, seed=4)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("page", [16, 48, 64, 128])
@pytest.mark.parametrize("lengths", [[1], [15, 16, 17], [0, 1, 2, 31, 32, 33], [1023, 5, 0, 257], [4099], [64] * 40])
def test_lengths_of_single_tokens(dtype, page, lengths):
    s = Setup(dtype, lengths, [1] * len(lengths), 2, 4, 128, page=page, seed=5)
    args = s.arguments()
    want = s.expected()
    check(lce.lce_kv_attention(*args[:5]), want)
    check(lce.lce_kv_attention(*args), want)


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 19), (False, 40), (True, 1000)])
def test_masks_of_several_tokens(dtype, causal, window):
    # sequences with no rows, with more rows than tokens (the first rows see nothing), with as many, with many before them
    s = Setup(dtype, [40, 7, 100, 0, 333, 16], [3, 12, 0, 4, 70, 16], 2, 3, 64, page=32, seed=6)
    check(lce.lce_kv_attention(*s.arguments(), causal=causal, window=window), s.expected(causal=causal, window=window))


@pytest.mark.parametrize("dtype,dim,group", [(BF16, 128, 4), (F16, 128, 1), (F32, 64, 2), (BF16, 256, 2), (BF16, 72, 5), (F32, 128, 4)])
@pytest.mark.parametrize("lengths,news", [([700], [700]), ([1300, 130], [200, 129]), ([257, 64, 300], [129, 64, 1])])
def test_prompts(dtype, dim, group, lengths, news):
    s = Setup(dtype, lengths, news, 1, group, dim, page=64, seed=7)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


def test_prompt_with_window_and_without_causality():
    s = Setup(BF16, [600, 450], [600, 100], 2, 2, 128, page=32, seed=8)
    check(lce.lce_kv_attention(*s.arguments(), window=100), s.expected(window=100))
    check(lce.lce_kv_attention(*s.arguments(), causal=False), s.expected(causal=False))


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("kv_heads,group,dim", [(6, 2, 40), (7, 8, 64), (5, 12, 128)])
def test_many_short_sequences(dtype, kv_heads, group, dim):
    """A warp to a sequence and head."""
    lengths = [(i * 37) % 70 for i in range(380)]
    s = Setup(dtype, lengths, [1] * len(lengths), kv_heads, group, dim, seed=40, table_extra=2)
    check(lce.lce_kv_attention(*s.arguments()[:5]), s.expected())
    s.table[5, 0], s.table[8, 1] = -1, s.desc.pages
    check(lce.lce_kv_attention(*s.arguments()[:5], window=30), s.expected(window=30, bad_tokens=[(5, slice(0, 16)), (8, slice(16, 32))]))


# shapes for which many rows are worth the tensor-core kernel: tables long enough, although not all of their sequences are
@pytest.mark.parametrize("dtype,dim", [(F16, 8), (BF16, 32), (F16, 40), (F16, 64), (BF16, 96), (F16, 100), (BF16, 128)])
def test_many_rows_of_every_head_size(dtype, dim):
    s = Setup(dtype, [700, 201, 130, 40], [300, 201, 3, 90], 2, 4, dim, page=48, seed=30, table_extra=200)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 77), (False, 300), (True, 1)])
def test_many_rows_masked(causal, window):
    s = Setup(BF16, [700, 20, 515, 0], [500, 64, 515, 40], 1, 8, 128, page=16, seed=31, table_extra=400)
    check(lce.lce_kv_attention(*s.arguments(), causal=causal, window=window), s.expected(causal=causal, window=window))


@pytest.mark.parametrize("dtype", [F16, BF16])
@pytest.mark.parametrize("scale", [None, -0.2, 0.0])
def test_many_rows_of_one_long_sequence_in_pieces(dtype, scale):
    s = Setup(dtype, [6001], [260], 1, 2, 128, page=128, seed=32, table_extra=900)
    args = s.arguments()
    got = lce.lce_kv_attention(*args, scale=scale)
    check(got, s.expected(scale=scale))
    assert torch.equal(got, lce.lce_kv_attention(*args, scale=scale))


@pytest.mark.parametrize("q_size", [1e-6, 40.0])
def test_many_rows_with_scales_that_grow_and_shrink(q_size):
    s = Setup(BF16, [900], [300], 2, 4, 64, page=32, seed=33, q_size=q_size, table_extra=300)
    grow = torch.exp2(torch.linspace(-40, 40, 900, dtype=torch.float64)).view(-1, 1, 1).to(DEV)
    for v in (s.v.double() * grow, s.v.double() * grow.flip(0)):
        s.v = v.to(BF16)
        s.store()
        check(lce.lce_kv_attention(*s.arguments()), s.expected())


def test_many_rows_and_what_is_not_a_number():
    s = Setup(F16, [800], [400], 2, 4, 128, page=64, seed=34, table_extra=200)
    s.k[650], s.v[700, 0, 40], s.v[701, 1, 100] = float("nan"), float("inf"), float("nan")  # seen by rows from 250, 300 and 301 on
    s.store()
    s.q[17, 3, 5], s.q[40, 0, 0] = float("inf"), float("nan")
    out, bound = s.expected()
    assert np.isfinite(out[:250][np.arange(250) != 17][:20]).all() and np.isnan(out[250:]).all()
    check(lce.lce_kv_attention(*s.arguments()), (out, bound))
    t = Setup(F16, [800], [400], 2, 4, 128, page=64, seed=34, table_extra=200)
    t.v[700, 0, 40], t.v[701, 1, 100] = float("inf"), float("nan")
    t.store()
    out, bound = t.expected()
    # a block of 32 channels of the value's own heads, from the first row that sees it on
    assert np.isnan(out[300:, :4, 32:64]).all() and np.isfinite(out[300:, :4, 64:]).all() and np.isfinite(out[:300]).all() and np.isnan(out[301:, 4:, 96:]).all()
    check(lce.lce_kv_attention(*t.arguments()), (out, bound))


def test_many_rows_strides_bad_pages_and_rows_of_no_sequence():
    s = Setup(BF16, [500, 333], [300, 200], 2, 4, 64, seed=35, table_extra=400)
    s.table[0, 3], s.table[1, 0] = -1, s.desc.pages
    want = s.expected(bad_tokens=[(0, slice(48, 64)), (1, slice(0, 16))])
    wide = torch.full((510, 3 * 8 * 64 + 5), 5.0, dtype=BF16, device=DEV)
    q = wide[:, 3:3 + 512].view(510, 8, 64)
    q[:500] = s.q
    args = s.arguments()
    args[1] = q
    back = torch.full((510, 8, 72), 9.0, dtype=BF16, device=DEV)
    lce.lce_kv_attention(*args, out=back[:, :, 8:])
    check(back[:500, :, 8:], want)
    assert (back[500:] == 9).all() and (back[:, :, :8] == 9).all()


def test_many_rows_captured_with_growing_sequences():
    s = Setup(BF16, [600, 400], [256, 256], 2, 4, 128, page=64, seed=36, table_extra=100)
    args = s.arguments()
    out, graph = torch.empty_like(s.q), torch.cuda.CUDAGraph()
    lce.lce_kv_attention(*args)
    with torch.cuda.graph(graph):
        lce.lce_kv_attention(*args, out=out)
    for lengths in ([600, 400], [300, 256], [10, 0], [599, 399]):
        args[4].copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        assert torch.equal(out, lce.lce_kv_attention(*args))
    args[4].copy_(torch.tensor([600, 400], dtype=torch.int32))
    graph.replay()
    check(out, s.expected())
    assert lce.lce_device_status() == 0


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_long_sequence_in_pieces(dtype):
    s = Setup(dtype, [20011, 3], [1, 1], 1, 2, 64, page=128, seed=9)
    args = s.arguments()
    got = lce.lce_kv_attention(*args)
    check(got, s.expected())
    for _ in range(3):
        assert torch.equal(got, lce.lce_kv_attention(*args))  # joined in a fixed order


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("q_size", [0.0, 1e-7, 30.0, 1e4])
def test_sharp_and_flat_weights(dtype, q_size):
    s = Setup(dtype, [500], [1], 2, 4, 64, seed=10, q_size=q_size)
    check(lce.lce_kv_attention(*s.arguments()), s.expected())
    check(lce.lce_kv_attention(*s.arguments(), scale=-0.3), s.expected(scale=-0.3))
    check(lce.lce_kv_attention(*s.arguments(), scale=0.0), s.expected(scale=0.0))


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_value_scales_that_grow_and_shrink_along_the_sequence(dtype):
    s = Setup(dtype, [400, 400], [1, 1], 1, 2, 64, seed=11)
    grow = torch.exp2(torch.linspace(-60, 60, 400, dtype=torch.float64)).view(-1, 1, 1).to(DEV)
    s.v = torch.cat([s.v[:400].double() * grow, s.v[400:].double() * grow.flip(0)]).to(dtype)
    s.k = s.k * 0.01
    s.store()
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
def test_infinities_and_nan_in_masked_places(dtype):
    """Tokens that a row does not see may hold anything: behind its position, in front of its window, behind the sequence's end."""
    s = Setup(dtype, [90, 60], [6, 1], 2, 2, 64, page=32, seed=12)
    s.k[89], s.v[88], s.v[89] = float("nan"), float("inf"), float("nan")  # seen by the last rows only
    s.k[2], s.v[3] = float("inf"), float("nan")                           # in front of the window of 50
    s.store()
    out, bound = s.expected(window=50)
    assert np.isfinite(out[:4]).all() and np.isnan(out[4:6]).all() and np.isfinite(out[6]).all()
    check(lce.lce_kv_attention(*s.arguments(), window=50), (out, bound))
    one = Setup(dtype, [40], [1], 1, 2, 64, seed=13)
    one.v[7, 0, 40] = float("inf")  # a block of 32 channels of the value
    one.store()
    got = lce.lce_kv_attention(*one.arguments())
    assert torch.isnan(got[:, :, 32:]).all()
    check(got, one.expected())


def test_rows_of_infinities_and_nan_stay_to_themselves():
    s = Setup(F16, [90, 90], [1, 1], 1, 4, 64, seed=14)
    want = s.expected()
    s.q[0, 1, 3], s.q[0, 2, 0] = float("inf"), float("nan")
    got = lce.lce_kv_attention(*s.arguments())
    assert torch.isnan(got[0, 1:3]).all()
    keep = np.array([[True, False, False, True], [True] * 4])
    check(got[torch.from_numpy(keep).to(DEV)], (want[0][keep], want[1][keep]))


def test_pages_outside_the_pool_are_masked():
    s = Setup(BF16, [100, 100], [1, 3], 1, 2, 64, seed=15)
    s.table[0, 2], s.table[1, 0], s.table[1, 6] = -1, s.desc.pages, 2 ** 31 - 1
    bad = [(0, slice(32, 48)), (1, slice(0, 16)), (1, slice(96, 100))]
    # the rows of sequence 1 stand on 97 .. 99: what they see ends with the page in front
    check(lce.lce_kv_attention(*s.arguments()), s.expected(bad_tokens=bad))
    s.table[:] = -1
    assert not lce.lce_kv_attention(*s.arguments()).any()


def test_lengths_past_the_table_end_with_it():
    s = Setup(BF16, [64, 64], [1, 1], 1, 2, 64, seed=16, table_extra=0)
    want = s.expected()
    s.lengths = [64, 1 << 30]
    check(lce.lce_kv_attention(*s.arguments(), causal=False), want)
    s.lengths = [64, -5]
    got = lce.lce_kv_attention(*s.arguments())
    check(got[:1], (want[0][:1], want[1][:1]))
    assert not got[1].any()


def test_strides_and_rows_of_no_sequence():
    s = Setup(BF16, [50, 70], [2, 3], 2, 2, 64, seed=17)
    want = s.expected()
    wide = torch.full((8, 3, 4, 67), 5.0, dtype=BF16, device=DEV)  # rows of 3 * 4 * 67, of which the q are a part
    q = wide[:, 1, :, 3:]
    q[:5] = s.q
    args = s.arguments()
    args[1] = q[:, :, :64]
    back = torch.full((8, 4, 70), 9.0, dtype=BF16, device=DEV)
    got = lce.lce_kv_attention(*args, out=back[:, :, 2:66])
    assert got.data_ptr() == back[:, :, 2:].data_ptr()
    check(back[:5, :, 2:66], want)
    assert (back[5:] == 9).all() and (back[:, :, :2] == 9).all() and (back[:, :, 66:] == 9).all()  # rows behind the last sequence stay
    flipped = s.q.transpose(0, 1).contiguous().transpose(0, 1)
    args[1] = flipped
    check(lce.lce_kv_attention(*args), want)


def test_streams_graphs_and_growing_sequences():
    s = Setup(BF16, [300, 20], [1, 1], 2, 4, 128, seed=18)
    args = s.arguments()
    room = torch.empty(lce.lce_kv_attention_workspace_bytes(s.desc, 2, 2, 8, args[3].shape[1], BF16), dtype=torch.uint8, device=DEV)
    first = lce.lce_kv_attention(*args[:5], workspace=room)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        again = lce.lce_kv_attention(*args[:5])
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(first, again)
    graph, out = torch.cuda.CUDAGraph(), torch.empty_like(s.q)
    with torch.cuda.graph(graph):
        lce.lce_kv_attention(*args[:5], out=out)
    room.random_(0, 255)
    other = torch.cuda.CUDAGraph()
    out2 = torch.empty_like(s.q)
    with torch.cuda.graph(other):  # a second graph with another workspace of its own
        lce.lce_kv_attention(*args[:5], out=out2, workspace=room)
    for lengths in ([300, 20], [17, 0], [1, 19], [299, 20]):
        args[4].copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        other.replay()
        t = Setup(BF16, [300, 20], [1, 1], 2, 4, 128, seed=18)
        for b, n in enumerate(lengths):
            keep = list(range(sum(t.lengths[:b]), sum(t.lengths[:b]) + n))
            q = t.q[b].double().cpu().numpy()
            (k, ks), (v, vs) = (ref.quantized(x[keep].double().cpu().numpy()) for x in (t.k, t.v))
            want = ref.attention(q, k, v, ks, vs, np.ones(n, bool), 128 ** -0.5, "bfloat16")
            check(out[b], want)
            assert torch.equal(out[b], out2[b])


def test_offsets_past_32_bits():
    d = lce.make_kv_desc(70000, 128, 4, 128)  # 5.2 GB
    cache = torch.empty(lce.lce_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
    s = Setup(BF16, [200], [1], 4, 2, 128, page=128, seed=19)
    s.desc, s.cache = d, cache
    s.table[0, :2] = [69999, 58300]
    t = np.arange(200)
    s.slots = [s.table[0][t // 128].astype(np.int64) * 128 + t % 128]
    s.store()
    check(lce.lce_kv_attention(*s.arguments()), s.expected())


def test_binding_refuses_what_does_not_fit():
    s = Setup(BF16, [50, 70], [1, 1], 2, 2, 64, seed=20)
    desc, q, cache, table, lengths, starts = s.arguments()
    good = dict(q=q, cache=cache, page_table=table, lengths=lengths)
    for change in (dict(q=q[:1]), dict(q=q.double()), dict(q=q[..., :32]), dict(q=q[:, :, ::2]), dict(cache=cache[16:]), dict(page_table=table[0]), dict(page_table=table.long()),
                   dict(lengths=lengths[:1]), dict(lengths=lengths.cpu()), dict(q_starts=starts[:2]), dict(window=-1), dict(out=q.float()), dict(out=q[:1]),
                   dict(workspace=torch.empty(16, device=DEV))):
        with pytest.raises(ValueError):
            lce.lce_kv_attention(desc, **{**good, **change})
    with pytest.raises(lce.LceError) as e:
        small = lce.lce_kv_attention_workspace_bytes(desc, 2, 2, 4, table.shape[1], BF16) - 1
        lce.lce_kv_attention(desc, **good, workspace=torch.empty(small, dtype=torch.uint8, device=DEV))
    assert e.value.status == 6
    with pytest.raises(lce.LceError) as e:
        lce.lce_kv_attention(desc, q[:, :3], cache, table, lengths)
    assert e.value.status == 1
