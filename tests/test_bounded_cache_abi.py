"""Host-side checks of rotary positions, attention weights by token and eviction: steps, sizes, refusals before anything is launched."""
import ctypes
import math
from decimal import Decimal, getcontext

import numpy as np
import pytest
import torch

import bounded_cache_reference as ref
import paper_2011_09398_b200 as lce
from paper_2011_09398_b200 import build as lce_build

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 6
FAKE = ctypes.c_void_p(4096)  # never dereferenced: the checks fail first
OFF_4, OFF_16 = ctypes.c_void_p(4098), ctypes.c_void_p(4104)


@pytest.fixture(scope="module")
def lib():
    lce_build.build()
    return lce.library()


# --- steps ---------------------------------------------------------------------------------------


def exact_frequencies(d, base, kind, factor=1.0, original=0.0, low=1.0, high=32.0):
    """In 60 digits."""
    getcontext().prec = 60
    pi = Decimal("3.14159265358979323846264338327950288419716939937510582097494")
    base, factor = Decimal(base), Decimal(factor)
    if kind == lce.ROTARY_BASE and d > 2:
        base *= factor ** (Decimal(d) / Decimal(d - 2))
    out = []
    for i in range(d // 2):
        f = base ** (Decimal(-2 * i) / Decimal(d))
        if kind == lce.ROTARY_LINEAR:
            f /= factor
        if kind == lce.ROTARY_PARTS:
            g = min(Decimal(1), max(Decimal(0), (Decimal(original) * f / (2 * pi) - Decimal(low)) / (Decimal(high) - Decimal(low))))
            f *= g + (1 - g) / factor
        out.append(f / (2 * pi))
    return out


@pytest.mark.parametrize("d", [0, 2, 4, 6, 64, 96, 128, 256])
@pytest.mark.parametrize("kind", [lce.ROTARY_PLAIN, lce.ROTARY_LINEAR, lce.ROTARY_BASE, lce.ROTARY_PARTS])
@pytest.mark.parametrize("base, factor", [(10000.0, 4.0), (500000.0, 8.0), (1.0, 1.0), (10000.0, 32.5)])
def test_steps(lib, d, kind, base, factor):
    steps = lce.lce_rotary_steps(d, base, kind, factor, 8192, 1.0, 32.0)
    assert steps.dtype == torch.int64 and steps.shape == (d // 2,)
    want = exact_frequencies(d, base, kind, factor, 8192)
    for s, w in zip(steps.tolist(), want):
        # fp64: the powers, two factors and the quotient are off by less than 2^-48 of themselves, and half a unit of 2^-64
        assert abs(Decimal(s % (1 << 64)) / Decimal(1 << 64) - w) <= w * Decimal(2) ** -48 + Decimal(2) ** -65


def test_steps_refusals(lib):
    room = (ctypes.c_uint64 * 200)()
    call = lambda d=64, kind=0, base=1e4, factor=2.0, original=100.0, low=1.0, high=32.0, to=room: lib.lce_rotary_steps(d, kind, base, factor, original, low, high, to)
    assert call() == 0
    for bad in (dict(d=-2), dict(d=3), dict(kind=-1), dict(kind=4), dict(base=0.5), dict(base=math.nan), dict(base=math.inf), dict(kind=1, factor=0.5), dict(kind=2, factor=math.nan),
                dict(kind=2, base=1e300, factor=1e300), dict(kind=3, original=0.0), dict(kind=3, low=-1.0), dict(kind=3, low=4.0, high=4.0), dict(kind=3, high=math.inf), dict(to=None)):
        assert call(**bad) == INVALID, bad
    assert call(d=258) == UNSUPPORTED
    with pytest.raises(lce.LceError):
        lce.lce_rotary_steps(7)


# --- rotary --------------------------------------------------------------------------------------


def rotary_desc(**change):
    fields = dict(head_dim=64, rotary_dim=32, layout=0, type=0, q_heads=4, k_heads=2, amplitude=1.0, tokens=3, q_token_stride=256, q_head_stride=64, k_token_stride=128,
                  k_head_stride=64, q_out_token_stride=256, q_out_head_stride=64, k_out_token_stride=128, k_out_head_stride=64)
    fields.update(change)
    return lce.RotaryDesc(**fields)


def test_rotary_refusals(lib):
    def call(d, q=FAKE, k=FAKE, positions=FAKE, steps=FAKE, q_out=FAKE, k_out=FAKE):
        return lib.lce_rotary(ctypes.byref(d), q, k, positions, steps, q_out, k_out, None)
    assert lib.lce_rotary(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == INVALID
    for bad in (dict(head_dim=0), dict(rotary_dim=-2), dict(rotary_dim=31), dict(rotary_dim=66), dict(layout=2), dict(layout=-1), dict(type=3), dict(q_heads=0), dict(k_heads=-1),
                dict(amplitude=math.nan), dict(amplitude=math.inf), dict(tokens=-1), dict(q_token_stride=-1), dict(k_out_head_stride=-64), dict(q_out_token_stride=1 << 40)):
        assert call(rotary_desc(**bad)) == INVALID, bad
    for bad in (dict(head_dim=257, rotary_dim=0), dict(q_heads=32768), dict(k_heads=32768), dict(tokens=1 << 31), dict(tokens=1 << 62), dict(tokens=(1 << 31) // 4)):
        assert call(rotary_desc(**bad)) == UNSUPPORTED, bad
    for name in ("q", "k", "positions", "steps", "q_out", "k_out"):
        assert call(rotary_desc(), **{name: None}) == INVALID, name
        assert call(rotary_desc(), **{name: OFF_4}) == ALIGNMENT, name
    assert call(rotary_desc(type=1), q=ctypes.c_void_p(4097)) == ALIGNMENT
    assert call(rotary_desc(), steps=ctypes.c_void_p(4100)) == ALIGNMENT
    assert call(rotary_desc(tokens=0), q=None, positions=None) == 0


# --- weights -------------------------------------------------------------------------------------


def weights_desc(**change):
    cache = lce.make_kv_desc(*change.pop("cache", (8, 16, 2, 64)))
    fields = dict(batch=2, heads=4, table_pages=3, type=0, causal=1, window=0, scale=0.125, decay=1.0, tokens=2, q_token_stride=256, q_head_stride=64,
                  previous_seq_stride=96, previous_head_stride=48, out_seq_stride=96, out_head_stride=48)
    fields.update(change)
    return lce.KvAttentionWeightsDesc(cache, **fields)


def weigh(lib, d, q=FAKE, cache=FAKE, table=FAKE, lengths=FAKE, starts=None, previous=None, out=FAKE, room=FAKE, size=1 << 40):
    return lib.lce_kv_attention_weights(ctypes.byref(d), q, cache, table, lengths, starts, previous, out, room, size, None)


def test_weights_refusals(lib):
    bytes_of = lambda d: lib.lce_kv_attention_weights_workspace_bytes(ctypes.byref(d))
    assert lib.lce_kv_attention_weights(None, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, FAKE, 1 << 40, None) == INVALID
    assert lib.lce_kv_attention_weights_workspace_bytes(None) == 0
    for bad in (dict(batch=0), dict(heads=0), dict(heads=3), dict(table_pages=0), dict(type=3), dict(type=-1), dict(causal=2), dict(window=-1), dict(tokens=-1),
                dict(scale=math.nan), dict(scale=math.inf), dict(decay=math.nan), dict(decay=-math.inf), dict(q_token_stride=-1), dict(previous_head_stride=-2), dict(out_seq_stride=1 << 40),
                dict(cache=(8, 20, 2, 64))):
        assert weigh(lib, weights_desc(**bad)) == INVALID, bad
        assert bytes_of(weights_desc(**bad)) == 0
    for bad in (dict(cache=(8, 16, 2, 257)), dict(table_pages=1 << 26), dict(tokens=1 << 30), dict(tokens=1 << 31), dict(tokens=1 << 62), dict(batch=1 << 20), dict(cache=((1 << 27) - 1, 16, 64, 64), heads=64)):
        assert weigh(lib, weights_desc(**bad), starts=FAKE) == UNSUPPORTED, bad
        assert bytes_of(weights_desc(**bad)) == 0
    d = weights_desc()
    for name in ("q", "cache", "table", "lengths", "out", "room"):
        assert weigh(lib, d, **{name: None}) == INVALID, name
    for name in ("q", "table", "lengths", "starts", "previous", "out"):
        assert weigh(lib, d, **{name: OFF_4}) == ALIGNMENT, name
    for name in ("cache", "room"):
        assert weigh(lib, d, **{name: OFF_16}) == ALIGNMENT, name
    assert weigh(lib, weights_desc(tokens=3)) == INVALID  # no q_starts: a row for each sequence
    for change in (dict(), dict(tokens=300), dict(tokens=300, type=1), dict(tokens=300, type=2, table_pages=100000)):
        d = weights_desc(**change)
        assert bytes_of(d) > 0 and weigh(lib, d, starts=FAKE, size=bytes_of(d) - 1) == WORKSPACE


# --- eviction ------------------------------------------------------------------------------------


def evict_desc(**change):
    cache = lce.make_kv_desc(*change.pop("cache", (8, 16, 2, 64)))
    fields = dict(batch=2, table_pages=3, kept_pages=2, budget=20, first=4, recent=8, scores_seq_stride=96, scores_head_stride=48, kept_scores_seq_stride=40, kept_scores_head_stride=20)
    fields.update(change)
    return lce.KvEvictDesc(cache, **fields)


def test_evict_refusals(lib):
    def call(d, cache=FAKE, table=FAKE, lengths=FAKE, scores=FAKE, kept_table=FAKE, kept=FAKE, kept_lengths=FAKE, kept_scores=FAKE):
        return lib.lce_kv_evict(ctypes.byref(d), cache, table, lengths, scores, kept_table, kept, kept_lengths, kept_scores, None)
    assert lib.lce_kv_evict(None, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == INVALID
    for bad in (dict(batch=0), dict(table_pages=0), dict(kept_pages=0), dict(budget=0), dict(budget=-5), dict(first=-1), dict(recent=-1), dict(first=13), dict(recent=17), dict(budget=33, first=0),
                dict(first=2 ** 31 - 1, recent=2 ** 31 - 1), dict(scores_seq_stride=-1), dict(kept_scores_head_stride=1 << 40), dict(cache=(8, 17, 2, 64))):
        assert call(evict_desc(**bad)) == INVALID, bad
    for bad in (dict(cache=(8, 16, 2, 257)), dict(table_pages=1 << 26), dict(kept_pages=1 << 26), dict(batch=65536), dict(cache=((1 << 27) - 1, 16, 64, 64))):
        assert call(evict_desc(**bad)) == UNSUPPORTED, bad
    for name in ("cache", "table", "lengths", "scores", "kept_table", "kept", "kept_lengths"):
        assert call(evict_desc(), **{name: None}) == INVALID, name
    for name in ("table", "lengths", "scores", "kept_table", "kept", "kept_lengths", "kept_scores"):
        assert call(evict_desc(), **{name: OFF_4}) == ALIGNMENT, name
    assert call(evict_desc(), cache=OFF_16) == ALIGNMENT


# --- binding -------------------------------------------------------------------------------------


def test_binding_refuses_cpu_tensors_and_wrong_shapes():
    d = lce.make_kv_desc(4, 16, 2, 32)
    cache, q, i32 = torch.zeros(lce.lce_kv_cache_bytes(d), dtype=torch.uint8), torch.zeros(1, 2, 32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_rotary(lce.make_rotary_desc(32), q, None, i32, lce.lce_rotary_steps(32))
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_kv_attention_weights(d, q, cache, i32.view(1, 1), i32)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_kv_evict(d, cache, i32.view(1, 1), i32, torch.zeros(1, 2, 16), i32.view(1, 1), 4)
    with pytest.raises(TypeError):
        lce.lce_rotary(d, q, None, i32, lce.lce_rotary_steps(32))
    with pytest.raises(TypeError):
        lce.lce_kv_evict(lce.make_rotary_desc(32), cache, i32.view(1, 1), i32, q, i32.view(1, 1), 4)


# --- the references by hand ------------------------------------------------------------------------


def test_reference_rotation_by_hand():
    x = np.array([[[1.0, 2.0, 3.0, 4.0, 5.0]]])
    quarter = 1 << 62
    out, met = ref.turned(x, [1], [quarter, 0], 4, False, 2.0)   # pairs (1, 3), (2, 4): the first by a quarter turn
    np.testing.assert_allclose(out[0, 0], [-6.0, 4.0, 2.0, 8.0, 5.0], atol=1e-12)
    np.testing.assert_allclose(met[0, 0], [8.0, 12.0, 8.0, 12.0, 0.0])
    out, _ = ref.turned(x, [-1], [quarter, quarter], 4, True, 1.0)  # pairs (1, 2), (3, 4), back
    np.testing.assert_allclose(out[0, 0], [2.0, -1.0, 4.0, -3.0, 5.0], atol=1e-12)


def test_reference_eviction_by_hand():
    scores = np.array([0.5, np.nan, 0.25, 0.5, -np.inf, 0.25, 9.0])
    valid = np.ones(7, bool)
    assert ref.kept(scores, 7, valid, 7, 0, 0).tolist() == [0, 1, 2, 3, 4, 5, 6]
    assert ref.kept(scores, 7, valid, 4, 0, 0).tolist() == [0, 2, 3, 6]   # of two alike the earlier
    assert ref.kept(scores, 7, valid, 4, 2, 1).tolist() == [0, 1, 3, 6]   # the first two, the last, and one more
    assert ref.kept(scores, 7, valid, 6, 0, 0).tolist() == [0, 2, 3, 4, 5, 6]  # NaN goes first
    valid[3] = False
    assert ref.kept(scores, 7, valid, 3, 0, 0).tolist() == [0, 2, 6]


def test_reference_weights_by_hand():
    k = np.zeros((3, 1, 32))
    k[1, 0, 0] = 1.0
    q = np.zeros((2, 2, 32))
    q[:, 1, 0] = np.log(3.0)
    shown = np.array([[True, True, False], [True, True, True]])
    out, bound = ref.weights(q, k, np.ones((3, 1, 1)), shown, 1.0)
    np.testing.assert_allclose(out[0], [1 / 2 + 1 / 3 + 1 / 4 + 1 / 5, 1 / 2 + 1 / 3 + 3 / 4 + 3 / 5, 1 / 3 + 1 / 5])
    assert (bound < 1e-4).all()
