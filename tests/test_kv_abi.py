"""Host-side checks of the key/value cache, its attention and the residual norm: sizes, refusals before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from paper_2011_09398_b200 import build as lce_build

INVALID, UNSUPPORTED, ALIGNMENT, WORKSPACE = 1, 2, 3, 6
FAKE, ODD = ctypes.c_void_p(4096), ctypes.c_void_p(4097)  # never dereferenced: the checks fail first


@pytest.fixture(scope="module")
def lib():
    lce_build.build()
    return lce.library()


def test_cache_bytes(lib):
    # 16 tokens of a head: (64 + 64 + 16) words for every 32 channels
    assert lce.lce_kv_cache_bytes(lce.make_kv_desc(3, 32, 5, 128)) == 3 * 2 * 5 * 4 * 144 * 4
    assert lce.lce_kv_cache_bytes(lce.make_kv_desc(1, 16, 1, 1)) == 144 * 4
    assert lce.lce_kv_cache_bytes(lce.make_kv_desc(100000, 128, 16, 256)) == 100000 * 8 * 16 * 8 * 144 * 4  # past 32 bits
    for bad in ((0, 16, 1, 64), (1, 0, 1, 64), (1, 24, 1, 64), (1, 8, 1, 64), (1, 16, 0, 64), (1, 16, 1, 0), (1, 16, 1, 257), (1 << 27, 16, 1, 64), (-1, 16, 1, 64)):
        assert lce.lce_kv_cache_bytes(lce.make_kv_desc(*bad)) == 0
    assert lib.lce_kv_cache_bytes(None) == 0


def test_quantize_and_dequantize_refusals(lib):
    d = lce.make_kv_desc(4, 16, 2, 64)
    r = ctypes.byref(d)
    assert lib.lce_kv_quantize(None, FAKE, FAKE, 0, 1, 128, 64, 128, 64, FAKE, FAKE, None) == INVALID
    for missing in range(4):
        k, v, s, c = (None if i == missing else FAKE for i in range(4))
        assert lib.lce_kv_quantize(r, k, v, 0, 1, 128, 64, 128, 64, s, c, None) == INVALID
    for kind in (-1, 3):
        assert lib.lce_kv_quantize(r, FAKE, FAKE, kind, 1, 128, 64, 128, 64, FAKE, FAKE, None) == INVALID
        assert lib.lce_kv_dequantize(r, FAKE, FAKE, 1, kind, FAKE, FAKE, None) == INVALID
    assert lib.lce_kv_quantize(r, FAKE, FAKE, 0, -1, 128, 64, 128, 64, FAKE, FAKE, None) == INVALID
    assert lib.lce_kv_quantize(r, FAKE, FAKE, 0, 1, -1, 64, 128, 64, FAKE, FAKE, None) == INVALID
    assert lib.lce_kv_quantize(r, FAKE, FAKE, 0, 1 << 31, 128, 64, 128, 64, FAKE, FAKE, None) == UNSUPPORTED
    assert lib.lce_kv_quantize(r, None, None, 0, 0, 128, 64, 128, 64, None, None, None) == 0  # no tokens: a no-op
    assert lib.lce_kv_quantize(r, ODD, FAKE, 1, 1, 128, 64, 128, 64, FAKE, FAKE, None) == ALIGNMENT
    assert lib.lce_kv_quantize(r, FAKE, FAKE, 1, 1, 128, 64, 128, 64, FAKE, ctypes.c_void_p(4104), None) == ALIGNMENT
    assert lib.lce_kv_dequantize(r, FAKE, FAKE, 1, 0, None, None, None) == INVALID
    assert lib.lce_kv_dequantize(r, FAKE, None, 1, 0, FAKE, FAKE, None) == INVALID
    assert lib.lce_kv_dequantize(r, FAKE, FAKE, -1, 0, FAKE, FAKE, None) == INVALID
    assert lib.lce_kv_dequantize(r, FAKE, FAKE, 1, 0, FAKE, ctypes.c_void_p(4098), None) == ALIGNMENT
    assert lib.lce_kv_dequantize(r, None, None, 0, 0, None, None, None) == 0
    for wrong, status in (((1, 17, 1, 64), INVALID), ((1, 16, 1, 300), UNSUPPORTED)):
        b = ctypes.byref(lce.make_kv_desc(*wrong))
        assert lib.lce_kv_quantize(b, FAKE, FAKE, 0, 1, 128, 64, 128, 64, FAKE, FAKE, None) == status
        assert lib.lce_kv_dequantize(b, FAKE, FAKE, 1, 0, FAKE, FAKE, None) == status


def attention_desc(**change):
    cache = lce.make_kv_desc(*change.pop("cache", (8, 16, 2, 64)))
    fields = dict(batch=2, heads=4, table_pages=3, type=0, causal=1, window=0, scale=0.125, tokens=2, q_token_stride=256, q_head_stride=64,
                  out_token_stride=256, out_head_stride=64)
    fields.update(change)
    return lce.KvAttentionDesc(cache, **fields)


def attend(lib, d, q=FAKE, cache=FAKE, table=FAKE, lengths=FAKE, starts=None, out=FAKE, room=FAKE, size=1 << 40):
    return lib.lce_kv_attention(ctypes.byref(d), q, cache, table, lengths, starts, out, room, size, None)


def test_attention_refusals(lib):
    assert lib.lce_kv_attention(None, FAKE, FAKE, FAKE, FAKE, None, FAKE, FAKE, 1 << 40, None) == INVALID
    for change in (dict(batch=0), dict(heads=0), dict(heads=3), dict(table_pages=0), dict(type=3), dict(type=-1), dict(causal=2), dict(window=-1), dict(tokens=-1),
                   dict(scale=float("nan")), dict(scale=float("inf")), dict(q_token_stride=-1), dict(out_head_stride=-2), dict(cache=(8, 20, 2, 64))):
        assert attend(lib, attention_desc(**change)) == INVALID, change
        assert lib.lce_kv_attention_workspace_bytes(ctypes.byref(attention_desc(**change))) == 0
    for change in (dict(cache=(8, 16, 2, 257)), dict(table_pages=1 << 27), dict(tokens=1 << 30), dict(batch=1 << 20)):
        assert attend(lib, attention_desc(**change), starts=FAKE) == UNSUPPORTED, change
    d = attention_desc()
    for name in ("q", "cache", "table", "lengths", "out", "room"):
        assert attend(lib, d, **{name: None}) == INVALID, name
    for name in ("q", "table", "lengths", "starts", "out"):
        assert attend(lib, d, **{name: ctypes.c_void_p(4098)}) == ALIGNMENT, name
    for name in ("cache", "room"):
        assert attend(lib, d, **{name: ctypes.c_void_p(4104)}) == ALIGNMENT, name
    size = lib.lce_kv_attention_workspace_bytes(ctypes.byref(d))
    assert size > 0 and attend(lib, d, size=size - 1) == WORKSPACE
    assert attend(lib, attention_desc(tokens=3)) == INVALID  # no q_starts: a row for each sequence
    assert attend(lib, attention_desc(tokens=0), q=None, starts=FAKE) == 0


def norm_desc(**change):
    fields = dict(rows=2, channels=64, post_norm=1, pre_norm=2, gate_activation=0, eps=1e-5, residual_scale=1.0, stream_type=0, type=0, x_stride=64,
                  branch_stride=64, gate_stride=0, y_stride=64, normed_stride=64)
    fields.update(change)
    return lce.ResidualNormDesc(**fields)


def test_residual_norm_refusals(lib):
    def call(d, x=FAKE, branch=FAKE, gate=None, post_weight=None, y=FAKE, normed=None, packed=None):
        return lib.lce_residual_norm(ctypes.byref(d), x, branch, gate, post_weight, None, None, None, y, normed, packed, None)
    assert lib.lce_residual_norm(None, FAKE, FAKE, None, None, None, None, None, FAKE, None, None, None) == INVALID
    for change in (dict(rows=-1), dict(channels=0), dict(post_norm=3), dict(pre_norm=-1), dict(gate_activation=lce.ACT_RELU), dict(type=3), dict(stream_type=-1),
                   dict(eps=-1.0), dict(eps=float("nan")), dict(residual_scale=float("inf")), dict(x_stride=-64), dict(y_stride=63)):
        assert call(norm_desc(**change)) == INVALID, change
    for change in (dict(channels=16385, y_stride=20000), dict(stream_type=1, type=2), dict(stream_type=1, type=0), dict(rows=1 << 31)):
        assert call(norm_desc(**change)) == UNSUPPORTED, change
    assert call(norm_desc(normed_stride=0), y=None, normed=FAKE) == INVALID
    assert call(norm_desc(), y=None) == INVALID  # nothing wanted
    assert call(norm_desc(), x=None) == INVALID
    assert call(norm_desc(), branch=None) == INVALID  # a norm of nothing
    assert call(norm_desc(post_norm=0), branch=None, gate=FAKE) == INVALID
    assert call(norm_desc(post_norm=0), branch=None, post_weight=FAKE) == INVALID
    assert call(norm_desc(rows=0), x=None) == 0
    for name in ("x", "branch", "gate", "post_weight", "y", "normed", "packed"):
        assert call(norm_desc(), **{name: ctypes.c_void_p(4098)}) == ALIGNMENT, name
    # a convolution knows no sigmoid
    conv = lce.make_desc(1, 4, 4, 32, 32, activation=lce.ACT_SIGMOID)
    assert lib.lce_bconv2d(ctypes.byref(conv), FAKE, FAKE, FAKE, FAKE, None, FAKE, None) == INVALID


def test_binding_refuses_cpu_tensors():
    d = lce.make_kv_desc(2, 16, 2, 32)
    cache, kv, slots = torch.zeros(lce.lce_kv_cache_bytes(d), dtype=torch.uint8), torch.zeros(1, 2, 32), torch.zeros(1, dtype=torch.int32)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_kv_quantize(d, kv, kv, slots, cache)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_kv_dequantize(d, cache, slots)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_kv_attention(d, kv, cache, slots.view(1, 1), slots)
    with pytest.raises(ValueError, match="CUDA"):
        lce.lce_residual_norm(lce.make_norm_desc(1, 32), torch.zeros(1, 32), torch.zeros(1, 32), y=torch.zeros(1, 32))
    with pytest.raises(TypeError):
        lce.lce_kv_quantize(lce.make_norm_desc(1, 32), kv, kv, slots, cache)


def test_reference_quantiser_by_hand():
    x = np.zeros((1, 40))
    x[0, :4] = [7.0, 2.5, -3.5, 0.49]
    x[0, 32:35] = [0.875, -0.0625, 0.1875]
    values, scales = ref.quantized(x)
    np.testing.assert_array_equal(scales, [[1.0, 0.125]])
    np.testing.assert_array_equal(values[0, :4], [7.0, 2.0, -4.0, 0.0])    # ties go to the even code
    np.testing.assert_array_equal(values[0, 32:35], [0.875, 0.0, 0.25])
    values, scales = ref.quantized(np.full((1, 1), 1.0))
    assert scales[0, 0] * 7 >= 1.0 > (scales[0, 0] - 2.0 ** -10) * 7 and scales[0, 0] == float(torch.tensor(scales[0, 0]).to(torch.bfloat16))
