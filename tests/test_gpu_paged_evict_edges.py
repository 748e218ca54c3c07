"""Eviction at both sides of every length and number of moves at which its kernels change, against the oracle's order."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H
from tests.test_gpu_paged_evict import check

pytestmark = pytest.mark.gpu
BF16 = ckv.BF16


@pytest.mark.parametrize("ties", [False, True])
@pytest.mark.parametrize("n", [256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097, 8192, 8193, 32768, 32769])
def test_slots_of_a_head(lib, n, ties):
    """One slot leaves, half of them do, nearly all."""
    gen = torch.Generator().manual_seed(n)
    cache = H.Cache(gen, BF16, 1, 1, 64, 64, [n], [n])
    w = cache.weight[0, 0, 0, :n]
    w[:] = (torch.rand(n, generator=gen) * 3).floor() if ties else torch.randn(n, generator=gen).mul(2).exp()
    for budget, recent in ((n - 1, 30), (n // 2, n // 8), (3, 0)):
        check(cache, [budget], recent)


@pytest.mark.parametrize("budget", [255, 256, 257, 300])
def test_moves_of_a_head(lib, budget):
    """Up to 256 slots move in the selecting workgroup, more in a launch of their own: here all that a head can move do, or few."""
    gen = torch.Generator().manual_seed(budget)
    n = 2 * budget + 7
    cache = H.Cache(gen, BF16, 2, 2, 64, 16, [n, n], [n, n], layers=2)
    slot = torch.arange(n)
    cache.weight[:, 0, :, :n] = (slot >= n - budget).float() + 0.25 * torch.rand(n, generator=gen)   # the last ones stay
    cache.weight[:, 1, :, :n] = (slot < budget).float()                                             # the first ones, nothing moves
    check(cache, [budget, budget], 0)
    check(cache, [budget, n - 2], 1)
