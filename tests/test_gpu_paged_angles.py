"""Sine and cosine of the rotation as they are, in rows of ones and zeros."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H
from tests.test_gpu_paged_append import call

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("d,rotary", [(64, 64), (128, 128), (128, 48)])
def test_sine_and_cosine(lib, d, rotary, inter):
    """A pair (1, 0) becomes (cos, sin).  The library's fp32 sine and cosine of a part of a revolution are off by a unit in the last place, 2^-24
    below one; the step back over the argument's rounding is rounded once, 2^-25, and its second order is below 2^-48: 1.5 * 2^-24, and
    0.1 for the double product (2^-34 of a revolution).  The argument's rounding alone would be another 1.6."""
    T = 3000
    gen = torch.Generator().manual_seed(d + rotary)
    cache = H.Cache(gen, ckv.F32, 1, 1, d, 16, [T], [0])
    i = torch.arange(rotary // 2)
    a, b = (2 * i, 2 * i + 1) if inter else (i, i + rotary // 2)
    qkv = torch.zeros((T, 3, d))
    qkv[..., a] = 1.0
    pos = torch.randint(0, 1 << 20, (T,), generator=gen).to(torch.int32)
    freq = (10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float()
    out = call(cache, [T], qkv, pos, None, None, freq, inter, cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(H.DEV), cache.len[0].to(H.DEV), None, None)
    angle = torch.remainder(pos.double()[:, None] * freq.double(), 2 * torch.pi)
    got = out[:, 0].cpu().double()
    assert float((got[:, a] - torch.cos(angle)).abs().max()) <= 1.6 * 2.0 ** -24
    assert float((got[:, b] - torch.sin(angle)).abs().max()) <= 1.6 * 2.0 ** -24
    assert bool((got[:, rotary:] == 0).all())
