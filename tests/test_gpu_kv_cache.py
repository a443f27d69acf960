"""Quantising keys and values into the 4-bit cache and reading them back, against the definition in 64 bits.  A code is unique, so
what is read back is one rounding of a known number: compared exactly."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV

pytestmark = pytest.mark.gpu
TYPES = [torch.float32, torch.float16, torch.bfloat16]


def make(pages, page, heads, dim):
    d = lce.make_kv_desc(pages, page, heads, dim)
    return d, torch.full((lce.lce_kv_cache_bytes(d),), 0xA5, dtype=torch.uint8, device=DEV)


def rows(rng, tokens, heads, dim, dtype):
    x = rng.standard_normal((tokens, heads, dim)) * np.exp2(rng.integers(-12, 12, size=(tokens, heads, 1)))
    return torch.from_numpy(x).to(dtype).to(DEV)


def expected(x, dtype):
    return torch.from_numpy(ref.quantized(x.double().cpu().numpy())[0]).to(dtype)


def same(a, b):
    return torch.equal(torch.nan_to_num(a.cpu().float(), nan=1e38), torch.nan_to_num(b.float(), nan=1e38))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,heads,dim,page", [(1, 1, 1, 16), (1, 8, 128, 16), (16, 2, 64, 16), (33, 3, 8, 32), (37, 5, 80, 48), (5, 1, 31, 16), (9, 2, 33, 64),
                                                   (130, 4, 96, 16), (64, 2, 160, 128), (21, 3, 192, 16), (18, 1, 224, 32), (50, 2, 256, 16), (19, 7, 100, 16), (300, 2, 255, 16)])
def test_store_and_load(dtype, tokens, heads, dim, page):
    rng = np.random.default_rng(tokens * 1000 + dim)
    pages = -(-tokens // page) + 2
    d, cache = make(pages, page, heads, dim)
    slots = torch.from_numpy(rng.permutation(pages * page)[:tokens].astype(np.int32)).to(DEV)
    k, v = rows(rng, tokens, heads, dim, dtype), rows(rng, tokens, heads, dim, dtype)
    lce.lce_kv_quantize(d, k, v, slots, cache)
    for out_type in TYPES:
        gk, gv = lce.lce_kv_dequantize(d, cache, slots, out_type)
        assert same(gk, expected(k, out_type)) and same(gv, expected(v, out_type))
    order = torch.from_numpy(rng.integers(0, tokens, size=2 * tokens)).to(DEV)  # any order, repeats
    gk, gv = lce.lce_kv_dequantize(d, cache, slots[order], torch.float32)
    assert same(gk, expected(k, torch.float32)[order.cpu()]) and same(gv, expected(v, torch.float32)[order.cpu()])


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_of_whole_tiles_and_ends_inside_them(dtype):
    """Tokens one after the other in their pages, from inside a tile to inside a tile, then the rest around them."""
    rng = np.random.default_rng(5)
    d, cache = make(5, 32, 3, 128)
    k, v = rows(rng, 160, 3, 128, dtype), rows(rng, 160, 3, 128, dtype)
    slots = torch.arange(160, dtype=torch.int32, device=DEV)
    for part in (slice(5, 90), slice(0, 5), slice(90, 91), slice(91, 160)):
        lce.lce_kv_quantize(d, k[part], v[part], slots[part].contiguous(), cache)
    gk, gv = lce.lce_kv_dequantize(d, cache, slots, dtype)
    assert same(gk, expected(k, dtype)) and same(gv, expected(v, dtype))


def test_strided_views_and_unaligned_rows():
    rng = np.random.default_rng(6)
    for dim, lead in ((64, 0), (64, 1), (40, 3), (7, 2)):
        heads, tokens = 3, 23
        d, cache = make(3, 16, heads, dim)
        wide = rows(rng, tokens, 1, 3 * heads * dim + 5, torch.float16).view(tokens, -1)
        k = wide[:, lead:lead + heads * dim].view(tokens, heads, dim)
        v = wide[:, lead + heads * dim:lead + 2 * heads * dim].view(tokens, heads, dim).transpose(0, 1).contiguous().transpose(0, 1)  # heads outside
        slots = torch.arange(tokens, dtype=torch.int32, device=DEV) + 7
        lce.lce_kv_quantize(d, k, v, slots, cache)
        gk, gv = lce.lce_kv_dequantize(d, cache, slots, torch.float16)
        assert same(gk, expected(k, torch.float16)) and same(gv, expected(v, torch.float16))
    one = rows(rng, 1, 2, 32, torch.float32).expand(9, 2, 32)  # one row for all tokens
    d, cache = make(1, 16, 2, 32)
    slots = torch.arange(9, dtype=torch.int32, device=DEV)
    lce.lce_kv_quantize(d, one, one, slots, cache)
    assert same(lce.lce_kv_dequantize(d, cache, slots)[0], expected(one, torch.float32))


@pytest.mark.parametrize("dtype", TYPES)
def test_codes_next_to_ties_and_scales_next_to_their_steps(dtype):
    """Values at, just below and just above every tie and every multiple of seven scales, over the exponents of fp32."""
    values = []
    for e in (-149, -140, -133, -128, -126, -120, -101, -100, -99, -20, 0, 3, 60, 120):
        for m in (1.0, 1.0 + 2.0 ** -7, 1.5, 1.9921875, 1.3671875):
            s = np.float32(np.ldexp(m, e))
            ticks = np.float32([(i + 0.5) for i in range(7)]) * s
            row = np.concatenate([ticks, np.nextafter(ticks, np.float32(0)), np.nextafter(ticks, np.float32(np.inf)), -ticks]).astype(np.float32)
            for top in (np.float32(7) * s, np.nextafter(np.float32(7) * s, np.float32(0)), np.nextafter(np.float32(7) * s, np.float32(np.inf))):
                values.append(np.concatenate([[top], row, [0, 0, -top]])[:32])
    x = np.stack(values).astype(np.float32)[:, None, :]
    k = torch.from_numpy(x).to(dtype).to(DEV)
    d, cache = make(-(-len(x) // 16), 16, 1, 32)
    slots = torch.arange(len(x), dtype=torch.int32, device=DEV)
    lce.lce_kv_quantize(d, k, -k, slots, cache)
    gk, gv = lce.lce_kv_dequantize(d, cache, slots)
    want = expected(k, torch.float32)
    assert same(gk, want) and same(gv, torch.where(want == 0, want, -want))


@pytest.mark.parametrize("dtype", TYPES)
def test_zeros_infinities_and_nan(dtype):
    x = torch.zeros(4, 1, 96, dtype=dtype)
    x[1, 0, 40] = float("inf")
    x[2, 0, 95] = float("nan")
    x[3, 0, :3] = torch.tensor([-float("inf"), 1.0, -0.0])
    x[3, 0, 64] = 1.0
    x = x.to(DEV)
    d, cache = make(1, 16, 1, 96)
    slots = torch.tensor([3, 0, 15, 8], dtype=torch.int32, device=DEV)
    lce.lce_kv_quantize(d, x, x, slots, cache)
    want = expected(x, dtype)
    assert torch.isnan(want[1, 0, 32:64]).all() and not torch.isnan(want[1, 0, 64:]).any()
    for got in lce.lce_kv_dequantize(d, cache, slots, dtype):
        assert same(got, want)


def test_skipped_slots_change_nothing_and_read_as_zeros():
    rng = np.random.default_rng(9)
    d, cache = make(3, 16, 2, 72)
    everything = torch.arange(48, dtype=torch.int32, device=DEV)
    k, v = rows(rng, 48, 2, 72, torch.bfloat16), rows(rng, 48, 2, 72, torch.bfloat16)
    lce.lce_kv_quantize(d, k, v, everything, cache)
    before = cache.clone()
    out = torch.tensor([-1, 48, 2 ** 31 - 1, -2 ** 31, 49], dtype=torch.int32, device=DEV)
    lce.lce_kv_quantize(d, k[:5], v[:5], out, cache)
    assert torch.equal(cache, before)
    # one row in the middle: every other row stays
    lce.lce_kv_quantize(d, k[:3], v[:3], torch.tensor([-1, 21, 48], dtype=torch.int32, device=DEV), cache)
    gk, gv = lce.lce_kv_dequantize(d, cache, everything, torch.bfloat16)
    k2, v2 = k.clone(), v.clone()
    k2[21], v2[21] = k[1], v[1]
    assert same(gk, expected(k2, torch.bfloat16)) and same(gv, expected(v2, torch.bfloat16))
    gk, gv = lce.lce_kv_dequantize(d, cache, out, torch.float32, torch.full((5, 2, 72), 3.0, device=DEV), torch.full((5, 2, 72), 3.0, device=DEV))
    assert not gk.any() and not gv.any()
    empty = torch.empty(0, dtype=torch.int32, device=DEV)
    lce.lce_kv_quantize(d, k[:0], v[:0], empty, cache)
    assert lce.lce_kv_dequantize(d, cache, empty)[0].shape == (0, 2, 72)


def test_offsets_past_32_bits():
    d = lce.make_kv_desc(70000, 128, 4, 128)  # 5.2 GB
    cache = torch.empty(lce.lce_kv_cache_bytes(d), dtype=torch.uint8, device=DEV)
    assert cache.numel() > 2 ** 32
    rng = np.random.default_rng(2)
    slots = torch.tensor([0, 70000 * 128 - 1, 58254 * 128 + 5, 29127 * 128, 69999 * 128], dtype=torch.int32, device=DEV)
    k, v = rows(rng, 5, 4, 128, torch.bfloat16), rows(rng, 5, 4, 128, torch.bfloat16)
    lce.lce_kv_quantize(d, k, v, slots, cache)
    gk, gv = lce.lce_kv_dequantize(d, cache, slots, torch.bfloat16)
    assert same(gk, expected(k, torch.bfloat16)) and same(gv, expected(v, torch.bfloat16))


def test_binding_refuses_what_does_not_fit():
    d, cache = make(2, 16, 2, 32)
    k, slots = torch.zeros(3, 2, 32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    for bad in ((k.half(), k, slots, cache), (k, k[:2], slots, cache), (k, k, slots[:2], cache), (k, k, slots.long(), cache), (k, k, slots, cache[:-16]),
                (k.transpose(1, 2), k, slots, cache), (k.double(), k.double(), slots, cache), (k, k, slots.cpu(), cache), (k[..., ::2].repeat(1, 1, 2)[..., ::2], k, slots, cache)):
        with pytest.raises(ValueError):
            lce.lce_kv_quantize(d, *bad)
    with pytest.raises(ValueError):
        lce.lce_kv_dequantize(d, cache, slots, torch.float64)
    with pytest.raises(ValueError):
        lce.lce_kv_dequantize(d, cache, slots, torch.float32, torch.empty(2, 2, 32, device=DEV))
    with pytest.raises(lce.LceError) as e:
        lce.lce_kv_quantize(d, k, k, slots, torch.empty(cache.numel() + 8, dtype=torch.uint8, device=DEV)[8:])
    assert e.value.status == 3
