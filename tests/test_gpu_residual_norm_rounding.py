"""Outputs of the residual norm beside sign bits: one rounding from the 64-bit result."""
import pytest
import torch

import paper_2011_09398_b200 as lce
from gpu_util import DEV

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,step", [(torch.bfloat16, 2.0 ** -7), (torch.float16, 2.0 ** -10)])
@pytest.mark.parametrize("channels", [64, 1000, 4099])
def test_outputs_beside_sign_bits_are_rounded_once(dtype, step, channels):
    """y = z = 1 + u with u next to half a step of the type, so near that fp32 would hold the tie itself."""
    x = torch.ones(3, channels, dtype=dtype, device=DEV)
    weight = torch.full((channels,), step / 2, device=DEV)
    near = torch.tensor([0.0, 2.0 ** -40, -2.0 ** -40], device=DEV)[torch.arange(channels, device=DEV) % 3]
    desc = lce.make_norm_desc(3, channels, lce.NORM_NONE, lce.NORM_NONE)
    y, z = torch.empty_like(x), torch.empty_like(x)
    bits = torch.empty(3, (channels + 31) // 32, dtype=torch.int32, device=DEV)
    for odd in (0, 1):  # the tie's neighbours: an even and an odd number of steps
        x.fill_(1 + odd * step)
        lce.lce_residual_norm(desc, x, torch.ones_like(x), None, weight, near, y=y, normed=z, packed=bits)
        up = (near > 0) | ((near == 0) & bool(odd))
        want = torch.where(up, 1 + (odd + 1) * step, 1 + odd * step).to(dtype).expand(3, -1)
        assert torch.equal(y, want) and torch.equal(z, want) and not bits.any()
