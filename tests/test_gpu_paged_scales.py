"""Attention over pages where scales are large and logits far from zero: ranges without a slot, empty heads, equal weights."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H
from tests.test_gpu_paged_attention import check

pytestmark = pytest.mark.gpu
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16


def queries(gen, cache):
    """Queries that leave logits the size they have at the default scale, so that the bars on them hold."""
    q = torch.randn((cache.batch, cache.hq, cache.d), generator=gen)
    return (q * (cache.d ** -0.5 / cache.scale)).to(H.KIND[cache.dtype])


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("scale", [0.72, 1.0, 3.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (7, 1, 64), (20, 2, 64)])
def test_whole_ranges_missing(lib, dtype, hq, hkv, d, scale, weights):
    """The first ranges of a head, one amid it, its last one, and all of them lie on pages that are not there; some heads are empty."""
    gen = torch.Generator().manual_seed(d + hq)
    room = [3000, 900, 40, 700, 1500]
    cache = H.Cache(gen, dtype, hq, hkv, d, 16, room, room, scale=scale)
    cache.table[0, :64] = -1               # ranges are 1024 slots at most, and whole blocks
    cache.table[0, 104:120] = cache.n_pages
    cache.table[1, 56] = -1
    cache.table[3, :44] = -1
    q = queries(gen, cache)
    check(cache, q, cache.len[0].tolist(), weights)
    check(cache, q, [[0] * hkv, [900] * hkv, [0] * hkv, [700] * hkv, [max(0, 1500 - 1499 * h) for h in range(hkv)]], weights)


@pytest.mark.parametrize("scale", [1.0, 3.0])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("room", [300, 500, 960])
def test_heads_of_one_workgroup(lib, dtype, scale, room):
    gen = torch.Generator().manual_seed(room)
    cache = H.Cache(gen, dtype, 16, 8, 64, 16, [room] * 16, [room] * 16, scale=scale)
    cache.table[0, :] = -1
    cache.table[1, 1:] = -1
    cache.len[0, 2:5] = 0
    cache.len[0, 5] = 1
    for weights in (True, False):
        check(cache, queries(gen, cache), cache.len[0].tolist(), weights)


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("weights", [False, True])
def test_sixteen_heads_with_missing_ranges(lib, dtype, weights):
    gen = torch.Generator().manual_seed(3)
    cache = H.Cache(gen, dtype, 16, 1, 128, 256, [45000], [45000], scale=1.0)
    cache.table[0, 8:16] = -1
    check(cache, queries(gen, cache), cache.len[0].tolist(), weights)
