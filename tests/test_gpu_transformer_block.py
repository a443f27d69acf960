"""The operators as a binarized transformer block runs them: norm and LceQuantize, binary projections (LceBConv2d with a 1x1 filter
over the tokens), the 4-bit cache, attention over it, LceQuantize, a binary projection back, and the boundary to the next block;
a prompt first, then single tokens.  Every step is checked against its definition on the inputs that it had."""
import numpy as np
import pytest
import torch

import kv_reference as ref
import oracle
import paper_2011_09398_b200 as lce
from gpu_util import DEV, words_to_host
from test_gpu_kv_attention import check

pytestmark = pytest.mark.gpu
HEADS, KV_HEADS, DIM, WIDTH, PAGE = 6, 2, 32, 160, 16
QKV = (HEADS + 2 * KV_HEADS) * DIM


class Projection:
    def __init__(self, rng, cin, cout):
        self.cin, self.cout = cin, cout
        self.w = (2 * rng.integers(0, 2, size=(cout, 1, 1, cin)) - 1).astype(np.int8)
        self.mult, self.bias = (rng.random(cout) * 0.05 + 0.05).astype(np.float32), (0.1 * rng.standard_normal(cout)).astype(np.float32)
        self.plain = lce.pack_weights(torch.from_numpy(self.w).to(DEV))

    def __call__(self, bits):
        n = bits.shape[0]
        desc = lce.make_desc(n, 1, 1, self.cin, self.cout, (1, 1), padding=lce.PAD_VALID, weights_packed=1)
        packed = lce.lce_bconv2d_pack_weights(desc, self.plain)
        out = lce.lce_bconv2d(desc, bits.view(n, 1, 1, -1), packed, torch.from_numpy(self.mult).to(DEV), torch.from_numpy(self.bias).to(DEV)).view(n, self.cout)
        acc = oracle.bconv2d_acc(oracle.unpack_pm1(words_to_host(bits), self.cin).reshape(n, 1, 1, self.cin), self.w)
        np.testing.assert_array_equal(out.cpu().numpy(), oracle.transform_float(acc, self.mult, self.bias).reshape(n, self.cout))
        return out


def test_prompt_then_single_tokens():
    rng = np.random.default_rng(3)
    w = lambda: torch.from_numpy(1 + 0.2 * rng.standard_normal(WIDTH)).float().to(DEV)
    qkv, back = Projection(rng, WIDTH, QKV), Projection(rng, HEADS * DIM, WIDTH)
    post, first, second = w(), w(), w()
    batch, prompt = 3, [21, 16, 1]
    pages = 12
    desc = lce.make_kv_desc(pages, PAGE, KV_HEADS, DIM)
    cache = torch.full((lce.lce_kv_cache_bytes(desc),), 0xFF, dtype=torch.uint8, device=DEV)
    table = rng.permutation(pages).reshape(batch, -1).astype(np.int32)
    table_d = torch.from_numpy(table).to(DEV)
    keys = [np.zeros((0, KV_HEADS, DIM)) for _ in range(batch)]
    values = [k.copy() for k in keys]
    lengths = [0] * batch
    for step in range(4):
        news = prompt if step == 0 else [1] * batch
        tokens = sum(news)
        x = torch.from_numpy(rng.standard_normal((tokens, WIDTH))).float().to(DEV)
        bits = torch.empty(tokens, WIDTH // 32, dtype=torch.int32, device=DEV)
        lce.lce_residual_norm(lce.make_norm_desc(tokens, WIDTH, lce.NORM_NONE, lce.NORM_RMS), x, pre_weight=first, packed=bits)
        np.testing.assert_array_equal(words_to_host(bits), ref.packed(ref.normed(x.double().cpu().numpy(), "rms", first.cpu().numpy(), None, 1e-5)))
        row = qkv(bits)
        q = row[:, :HEADS * DIM].view(tokens, HEADS, DIM)
        k, v = (row[:, (HEADS + i * KV_HEADS) * DIM:(HEADS + (i + 1) * KV_HEADS) * DIM].view(tokens, KV_HEADS, DIM) for i in range(2))
        slots = np.concatenate([table[b][(lengths[b] + np.arange(n)) // PAGE] * PAGE + (lengths[b] + np.arange(n)) % PAGE for b, n in enumerate(news)])
        lce.lce_kv_quantize(desc, k, v, torch.from_numpy(slots.astype(np.int32)).to(DEV), cache)
        at = 0
        for b, n in enumerate(news):
            keys[b] = np.concatenate([keys[b], k[at:at + n].double().cpu().numpy()])
            values[b] = np.concatenate([values[b], v[at:at + n].double().cpu().numpy()])
            lengths[b] += n
            at += n
        starts = torch.tensor(np.concatenate([[0], np.cumsum(news)]), dtype=torch.int32, device=DEV)
        o = lce.lce_kv_attention(desc, q, cache, table_d, torch.tensor(lengths, dtype=torch.int32, device=DEV), starts if step == 0 else None)
        want, bound = np.zeros(o.shape), np.zeros(o.shape)
        at = 0
        for b, n in enumerate(news):
            (kq, ks), (vq, vs) = ref.quantized(keys[b]), ref.quantized(values[b])
            for i in range(n):
                shown = np.arange(lengths[b]) <= lengths[b] - n + i
                want[at], bound[at] = ref.attention(q[at].double().cpu().numpy(), kq, vq, ks, vs, shown, DIM ** -0.5, "float32")
                at += 1
        check(o, (want, bound))
        o_bits = lce.lce_bitpack(o.view(tokens, HEADS * DIM))
        np.testing.assert_array_equal(words_to_host(o_bits), oracle.bitpack(o.view(tokens, -1).cpu().numpy()))
        branch = back(o_bits)
        y, next_bits = torch.empty_like(x), torch.empty_like(bits)
        lce.lce_residual_norm(lce.make_norm_desc(tokens, WIDTH, lce.NORM_RMS, lce.NORM_RMS, residual_scale=0.5), x, branch, None, post, None, second, None, y, None, next_bits)
        u = ref.normed(branch.double().cpu().numpy(), "rms", post.cpu().numpy(), None, 1e-5)
        y64 = x.double().cpu().numpy() + 0.5 * u
        # fp32: two sums of 14 levels of roundings and a dozen more, of 2^-24 of what meets in a value each
        assert (np.abs(y.double().cpu().numpy() - y64) <= 2.0 ** -18 * (np.abs(x.double().cpu().numpy()) + 0.5 * np.abs(u))).all()
        np.testing.assert_array_equal(words_to_host(next_bits), ref.packed(ref.normed(y64, "rms", second.cpu().numpy(), None, 1e-5)))
