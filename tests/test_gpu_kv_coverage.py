"""That attention over the 4-bit cache counts every token once, and that its kernel for few rows cuts and joins sequences of every
form: results that depend on each token alone, and all the ways in which pieces meet."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import BF16, F16, F32, NAMES, Setup, check

pytestmark = pytest.mark.gpu


def room(s, one_row):
    """Bytes of the workspace; 16 where no sequence can be in pieces."""
    tokens = len(s.news) if one_row else sum(s.news)
    return lce.lce_kv_attention_workspace_bytes(s.desc, len(s.lengths), tokens, s.kv_heads * s.group, s.table.shape[1], s.dtype)


@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 5000), (False, 3000)])
@pytest.mark.parametrize("dtype,kv_heads,group,dim,lengths,news", [
    (BF16, 2, 4, 128, [9001, 5000, 30], [1, 1, 1]),      # up to 16 pieces, a warp joins a column
    (F32, 1, 2, 64, [9001, 1100], [1, 1]),
    (F16, 2, 5, 96, [9001, 2500], [3, 8]),               # 16 columns, several rows
    (F32, 2, 5, 40, [9001, 0, 2500], [9, 4, 1]),
    (BF16, 1, 3, 256, [9500], [5]),                      # more than 128 channels
    (F32, 1, 4, 192, [10000, 700], [7, 2]),
    (F16, 1, 20, 160, [20000], [1]),                     # more than 16 pieces, three tiles of columns
    (BF16, 1, 20, 128, [20000, 40], [1, 1]),
])
def test_pieces_of_every_form(dtype, kv_heads, group, dim, lengths, news, causal, window):
    s = Setup(dtype, lengths, news, kv_heads, group, dim, page=64, seed=60)
    if not window:
        assert room(s, False) > 16
    args, want = s.arguments(), s.expected(causal=causal, window=window)
    got = lce.lce_kv_attention(*args, causal=causal, window=window)
    check(got, want)
    assert torch.equal(got, lce.lce_kv_attention(*args, causal=causal, window=window))
    if news == [1] * len(news):
        check(lce.lce_kv_attention(*args[:5], causal=causal, window=window), want)


# (sequences, rows): clusters, warps alone, pieces (few and many), several rows, and many rows in one and in several pieces
FORMS = {"cluster": ([777], [1], 2, 4, 0), "short": ([70] * 300, [1] * 300, 4, 2, 0), "few pieces": ([9001, 700], [1, 1], 1, 4, 0), "pieces": ([20011], [1], 1, 2, 0),
         "several rows": ([600, 333], [5, 3], 2, 4, 0), "many rows": ([900], [300], 2, 4, 60), "many rows in pieces": ([6001], [260], 1, 2, 900)}


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [64, 128, 192])
@pytest.mark.parametrize("form", list(FORMS))
def test_every_token_counts_once(dtype, dim, form):
    """Equal weights (q = 0), and values that are 0 but for one channel of one token: the result there is that value over the number of
    tokens.  One call tells as many tokens as there are channels; the tokens at the edges of tiles and pages are gone through."""
    lengths, news, kv_heads, group, extra = FORMS[form]
    s = Setup(dtype, lengths, news, kv_heads, group, dim, page=64, seed=61, q_size=0.0, table_extra=extra)
    args, total, per_call = s.arguments(), sum(lengths), kv_heads * dim
    t = torch.arange(total, device=DEV)
    if total > 2000:  # the edges
        t = t[(t % 16 == 0) | (t % 16 == 15)]
    first = np.concatenate([[0], np.cumsum(lengths)])
    rows = np.concatenate([[0], np.cumsum(news)])
    owner = torch.from_numpy(np.searchsorted(first, t.cpu().numpy(), side="right") - 1).to(DEV)
    # A value of 7 has code 7 and scale 1, the rest of its block 0.  The weight of a token is 1 / n to 2^-11 (its f16; for fp32 rows 2^-21) and the
    # sums' steps; 16-bit rows: products cut by at most 34 * 2^-15 of the steps of the 32 values that share the block, 32 / 7 of the value.
    n = float(max(lengths))
    off = ref.HALF_STEP[NAMES[dtype]] + (n / 16 + 65) * 2.0 ** -23 + (2.0 ** -21 if dtype == F32 else 2.0 ** -11 + 34 * 2.0 ** -15 * 32 / 7)
    assert off < 0.05
    for at in range(0, t.numel(), per_call):
        some, own = t[at:at + per_call], owner[at:at + per_call]
        place = torch.arange(some.numel(), device=DEV)
        s.v = torch.zeros(total, kv_heads, dim, dtype=dtype, device=DEV)
        s.v[some, place // dim, place % dim] = 7
        s.store()
        got = lce.lce_kv_attention(*args, causal=False).double()
        want = torch.zeros_like(got)
        for b in torch.unique(own).tolist():
            mine = place[own == b]
            for g in range(group):
                want[rows[b]:rows[b + 1], mine // dim * group + g, mine % dim] = 7.0 / lengths[b]
        # everything else is 0 but for what the block's other values may leave
        other = 0.0 if dtype == F32 else 34 * 2.0 ** -15 * 32
        assert bool((got - want).abs().le(torch.where(want > 0, want * off, other / min(n for n in lengths if n))).all()), (at, (got - want).abs().max())


@pytest.mark.parametrize("dtype", [F32, F16, BF16])
@pytest.mark.parametrize("dim,group", [(64, 2), (128, 4), (256, 1)])
def test_one_token_that_takes_all_the_weight(dtype, dim, group):
    """Its key lies along q, with a score 40 above all others: the result is its value as it is stored."""
    at = [0, 1, 15, 16, 17, 31, 127, 128, 640, 1023, 1024, 1039, 1040, 1087, 1088, 1098]  # of 1099 tokens
    s = Setup(dtype, [1099] * len(at), [1] * len(at), 1, group, dim, page=64, seed=62)
    s.q.fill_(1.0)
    s.k = torch.zeros_like(s.k)
    for b, token in enumerate(at):
        s.k[b * 1099 + token] = 40 * dim ** -0.5
    s.store()
    got = lce.lce_kv_attention(*s.arguments()[:5]).double().cpu().numpy()
    values, scales = ref.quantized(s.v.double().cpu().numpy())
    hot = np.arange(len(at)) * 1099 + at
    out = values[hot]  # [sequence][1][dim]
    # the others' weight is 1098 e^-39.8 < 1e-14; keys are rounded to 4 bits, which keeps 40 as a code of 7 of its own scale (8 bits)
    step = np.repeat(scales[hot], 32, -1)[:, :, :dim]
    most = np.abs(values).max()
    off = (ref.HALF_STEP[NAMES[dtype]] + (2.0 ** -21 if dtype == F32 else 2.0 ** -11) + 140 * 2.0 ** -23) * np.abs(out) + 1e-13 * most + \
          (0.0 if dtype == F32 else 34 * 2.0 ** -15 * step) + 2.0 ** -31 * 1099 * most
    assert (np.abs(got - out) <= off).all(), (np.abs(got - out) - off).max()
    assert (off < 0.5 * step).all()  # another token, or a code more or less, would be seen


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_thousands_of_sequences_of_all_lengths(dtype):
    """The search for a block's work goes through them 32 at a time: empty ones, some without rows, a long one among them in pieces."""
    rng = np.random.default_rng(63)
    lengths, news = rng.integers(0, 40, 4101).tolist(), rng.integers(0, 4, 4101).tolist()
    lengths[2600], news[2600], lengths[4100], news[4100] = 3000, 2, 17, 5
    s = Setup(dtype, lengths, news, 1, 2, 32, seed=63)
    assert room(s, False) > 16
    args = s.arguments()
    want = s.expected()
    check(lce.lce_kv_attention(*args), want)
    one = np.concatenate([[0], np.cumsum(news)])[:-1][np.array(news) > 0]  # the first row of each that has one, by itself
    keep = torch.from_numpy(one).to(DEV)
    has = torch.from_numpy(np.flatnonzero(np.array(news) > 0)).to(DEV)
    shorter = torch.tensor(np.array(lengths) - np.array(news) + 1, dtype=torch.int32, device=DEV)  # where that row stands last
    got = lce.lce_kv_attention(s.desc, s.q[keep], s.cache, args[3][has], shorter[has])
    check(got, (want[0][one], want[1][one]))
