"""Generating with a bounded cache, as a binarized transformer block runs it: binary projections (LceBConv2d with a 1x1 filter over the
tokens) write q, k and v side by side, rotary positions turn q and k where they lie, the keys and values go into the 4-bit cache,
attention reads it, the weights of every token add up, and once a sequence has passed its budget the least attended tokens of each head leave:
a prompt first, then single tokens.  Every step is checked against its definition on the inputs that it had."""
import numpy as np
import pytest
import torch

import bounded_cache_reference as bounded
import kv_reference as ref
import paper_2011_09398_b200 as lce
from gpu_util import DEV
from test_gpu_kv_attention import check
from test_gpu_transformer_block import Projection

pytestmark = pytest.mark.gpu
HEADS, KV_HEADS, DIM, WIDTH, PAGE, PART = 6, 2, 32, 160, 16, 24
QKV = (HEADS + 2 * KV_HEADS) * DIM
BUDGET, FIRST, RECENT, EVERY = 40, 2, 8, 6


def test_prompt_then_single_tokens():
    rng = np.random.default_rng(5)
    i32 = lambda a: torch.from_numpy(np.ascontiguousarray(a, np.int32)).to(DEV)
    qkv = Projection(rng, WIDTH, QKV)
    prompt, batch = [75, 33, 1], 3
    pages_each = 6
    pages = batch * pages_each * 2  # those that are read, and those that what stays moves to
    desc = lce.make_kv_desc(pages, PAGE, KV_HEADS, DIM)
    cache = torch.full((lce.lce_kv_cache_bytes(desc),), 0xFF, dtype=torch.uint8, device=DEV)
    order = rng.permutation(pages)
    tables = order.reshape(2, batch, pages_each).astype(np.int32)
    table = 0
    rotary = lce.make_rotary_desc(DIM, PART, lce.ROTARY_PAIRS)
    steps = lce.lce_rotary_steps(PART, scaling=lce.ROTARY_PARTS, factor=4.0, original_length=64, low_turns=1, high_turns=8)
    sums = torch.zeros(batch, KV_HEADS, pages_each * PAGE, device=DEV)
    rows = [dict(k=np.zeros((0, KV_HEADS, DIM)), ks=np.zeros((0, KV_HEADS, 1)), v=np.zeros((0, KV_HEADS, DIM)), vs=np.zeros((0, KV_HEADS, 1)), w=np.zeros((KV_HEADS, 0)),
                 wb=np.zeros((KV_HEADS, 0))) for _ in range(batch)]
    lengths, positions, evictions = np.zeros(batch, int), np.zeros(batch, int), 0
    for step in range(20):
        news = prompt if step == 0 else [1] * batch
        tokens = sum(news)
        bits = lce.lce_bitpack(torch.from_numpy(rng.standard_normal((tokens, WIDTH)).astype(np.float32)).to(DEV))
        row = qkv(bits)
        before = row.clone()
        view = lambda t, first, heads: t[:, first * DIM:(first + heads) * DIM].view(tokens, heads, DIM)
        q, k, v = view(row, 0, HEADS), view(row, HEADS, KV_HEADS), view(row, HEADS + KV_HEADS, KV_HEADS)
        # positions go on from where the sequence is, whatever the cache still holds of it
        at = np.concatenate([positions[b] + np.arange(n) for b, n in enumerate(news)])
        lce.lce_rotary(rotary, q, k, i32(at), steps.to(DEV), q, k)
        for got, heads, first in ((q, HEADS, 0), (k, KV_HEADS, HEADS)):
            want, met = bounded.turned(view(before, first, heads).double().cpu().numpy(), at, steps.tolist(), PART, True, 1.0)
            assert (np.abs(got.double().cpu().numpy() - want) <= bounded.turned_bound(want, met, "float32")).all()
        assert torch.equal(v, view(before, HEADS + KV_HEADS, KV_HEADS))
        slots = np.concatenate([tables[table][b][(lengths[b] + np.arange(n)) // PAGE] * PAGE + (lengths[b] + np.arange(n)) % PAGE for b, n in enumerate(news)])
        lce.lce_kv_quantize(desc, k, v, i32(slots), cache)
        token = 0
        for b, n in enumerate(news):
            for name, t in (("k", k), ("v", v)):
                values, scales = ref.quantized(t[token:token + n].double().cpu().numpy())
                rows[b][name], rows[b][name + "s"] = np.concatenate([rows[b][name], values]), np.concatenate([rows[b][name + "s"], scales])
            token, lengths[b], positions[b] = token + n, lengths[b] + n, positions[b] + n
        starts = i32(np.concatenate([[0], np.cumsum(news)])) if step == 0 else None
        call = (desc, q, cache, i32(tables[table]), i32(lengths), starts)
        o = lce.lce_kv_attention(*call)
        assert lce.lce_kv_attention_weights(*call, previous=sums, out=sums, decay=0.75) is sums
        want, bound = np.zeros(o.shape), np.zeros(o.shape)
        token = 0
        for b, n in enumerate(news):
            r = rows[b]
            shown = np.arange(lengths[b]) <= lengths[b] - n + np.arange(n)[:, None]
            rows_of_q = q[token:token + n].double().cpu().numpy()
            for i in range(n):
                want[token + i], bound[token + i] = ref.attention(rows_of_q[i], r["k"], r["v"], r["ks"], r["vs"], shown[i], DIM ** -0.5, "float32")
            w, wb = bounded.weights(rows_of_q, r["k"], r["ks"], shown, DIM ** -0.5)
            pad = np.zeros((KV_HEADS, n))
            r["w"] = w + 0.75 * np.concatenate([r["w"], pad], 1)
            r["wb"] = wb + 0.75 * np.concatenate([r["wb"], pad], 1) + 2.0 ** -23 * r["w"]
            got = sums[b, :, :lengths[b]].double().cpu().numpy()
            assert (np.abs(got - r["w"]) <= r["wb"]).all()
            token += n
        check(o, (want, bound))
        if step % EVERY:
            continue
        # every sequence moves, whether it has passed its budget or not; scores are what the library has, so the choice is exact
        scores = sums.cpu().numpy()
        kept, kept_lengths, _ = lce.lce_kv_evict(desc, cache, i32(tables[table]), i32(lengths), sums.clone(), i32(tables[1 - table]), BUDGET, FIRST, RECENT, kept_scores=sums)
        table, evictions = 1 - table, evictions + 1
        kept, new_lengths = kept.cpu().numpy(), kept_lengths.cpu().numpy()
        for b in range(batch):
            count = min(lengths[b], BUDGET)
            assert new_lengths[b] == count
            chosen = np.stack([bounded.kept(scores[b, h], lengths[b], np.ones(lengths[b], bool), BUDGET, FIRST, RECENT) for h in range(KV_HEADS)])
            assert np.array_equal(kept[b, :, :count], chosen)
            r = rows[b]
            for name in ("k", "ks", "v", "vs"):
                r[name] = np.stack([r[name][chosen[h], h] for h in range(KV_HEADS)], 1)
            for name in ("w", "wb"):
                r[name] = np.take_along_axis(r[name], chosen, 1)
            j = np.arange(count)
            back = lce.lce_kv_dequantize(desc, cache, i32(tables[table][b][j // PAGE] * PAGE + j % PAGE))
            for got, name in zip(back, "kv"):
                assert np.array_equal(got.double().cpu().numpy(), r[name])
            lengths[b] = count
    assert evictions == 4 and lengths[0] < positions[0]
