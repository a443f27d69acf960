"""Eviction where a block has many tokens to choose from: every form of the choice, by how many of a row's tokens a thread keeps, on which how many
blocks share a row follows from how many rows there are."""
import numpy as np
import pytest
import torch

from test_gpu_kv_evict import Pool

pytestmark = pytest.mark.gpu

# sequences, heads, tokens of the longest: 5 - 8 thousand of a block's own where there are more blocks than SMs (threads of sixteen tokens, 512 of
# them), or fewer (eight, 1024); 9 - 16 thousand (sixteen, 1024), one block, two or eight to a row
FORMS = [(19, 8, 4160), (19, 8, 8192), (150, 1, 5000), (2, 4, 65536), (3, 25, 20000), (1, 1, 131072), (1, 8, 131072), (30, 5, 9000), (75, 2, 16384)]


@pytest.mark.parametrize("kind", ["numbers", "few values", "nan and infinities"])
@pytest.mark.parametrize("sequences, kv_heads, most", FORMS)
def test_forms_of_the_choice(kind, sequences, kv_heads, most):
    rng = np.random.default_rng(most + sequences)
    lengths = [int(n) for n in rng.integers(0, most + 1, sequences)]
    lengths[-1] = most
    p = Pool(lengths, most // 4 + 5, kv_heads=kv_heads, dim=4, page=64, seed=most, more=0)
    s = p.scores
    if kind == "few values":
        s[:] = rng.integers(0, 3, s.shape)
    elif kind == "nan and infinities":
        s[rng.random(s.shape) < 0.5] = np.nan
        s[rng.random(s.shape) < 0.4] = -np.inf
        s[rng.random(s.shape) < 0.05] = np.inf
    kept, counts = p.check(first=3, recent=most // 16)
    assert counts.tolist() == [min(n, p.budget) for n in lengths]
    again = [t.cpu().numpy() for t in p.run(torch.from_numpy(s).to(p.cache.device), first=3, recent=most // 16)]
    assert np.array_equal(again[0], kept)
