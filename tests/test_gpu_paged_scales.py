"""Attention over pages where scales are large and logits far from zero: ranges without a slot, empty heads, equal weights."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H
from tests.test_gpu_paged_attention import LOGIT, PAIR, check, run

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


def far(gen, dtype, room, d, sign, far_k, far_q, every=1, scale=0.0):
    """A cache whose scores are sign * far_k * far_q in every so many-th slot and twice as far below zero, or half as far above, in the others."""
    cache = H.Cache(gen, dtype, 8, 2, d, 16, [room], [room], scale=scale)
    there = torch.isfinite(cache.k[0])
    cache.k[0][there] = 0
    _, page, row = cache.slots(0, 0, room)
    first = torch.full((room,), sign * far_k * (0.5 if sign > 0 else 2.0))
    first[::every] = sign * far_k
    cache.k[0, page, :, row, 0] = first[:, None].to(H.KIND[dtype])
    q = torch.zeros((1, 8, d), dtype=H.KIND[dtype])
    q[..., 0] = far_q
    return cache, q


def equal_shares(cache, q, every):
    """Every so many-th slot of a head gets the same part of every query head, the others nothing."""
    room = int(cache.len[0, 0, 0])
    n = -(-room // every)
    out, lse, weight = run(cache, q, None, torch.zeros_like(cache.weight[0]))
    # the reciprocal of n, off by a step of fp32 (two roundings), once per query head and added up: its sums of two and four are
    # exact, that of three and the one with what was there are rounded; the reference is the scores' own, so that their exponentials are 1
    want = torch.zeros(room)
    want[::every] = 4.0 / n
    assert float((weight[0, :, :room] - want).abs().max()) <= 5 * 2.0 ** -24 * 4.0 / n
    for h in range(2):
        _, v = cache.rows(cache.v, 0, h, room)
        v = v[::every]
        assert float((out[0, 4 * h:4 * h + 4].double() - v.mean(0)).abs().max()) <= PAIR * float(v.abs().max())
    return lse


@pytest.mark.parametrize("every", [1, 3])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("room", [200, 500, 900, 3000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_equal_keys_far_from_zero(lib, dtype, room, sign, every):
    """Logits of 2^24 and of 2^57: what a slot receives is not lost beside them."""
    far_k, far_q = (2.0 ** 13, 2.0 ** 14) if dtype == F16 else (2.0 ** 30, 2.0 ** 30)
    gen = torch.Generator().manual_seed(room)
    cache, q = far(gen, dtype, room, 64, sign, far_k, far_q, every)
    lse = equal_shares(cache, q, every)
    logit = sign * far_k * far_q / 8
    assert float((lse.double() - logit).abs().max()) <= 4 * 2.0 ** -24 * abs(logit) + 10


@pytest.mark.parametrize("every", [1, 3])
@pytest.mark.parametrize("sign", [1.0, -1.0])
@pytest.mark.parametrize("room", [200, 900, 3000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_logits_at_the_ends_of_fp32(lib, dtype, room, sign, every):
    """Logits of up to 255 / 128 * 2^127 in magnitude, finite as they are and not in units of log2 e."""
    far_k = 1.9921875 * 2.0 ** 63 * (1.0 if sign > 0 or every == 1 else 0.5)
    gen = torch.Generator().manual_seed(room)
    cache, q = far(gen, dtype, room, 128, sign, far_k, 2.0 ** 64, every, scale=1.0)
    lse = equal_shares(cache, q, every)
    logit = sign * far_k * 2.0 ** 64
    assert bool(torch.isfinite(lse).all()) and float((lse.double() - logit).abs().max()) <= 4 * 2.0 ** -24 * abs(logit)


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("room", [200, 900, 3000])
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_scales_at_the_end_of_fp32(lib, dtype, room, weights):
    """A scale that is finite as it is and not in units of log2 e: the largest score has all the weight; missing pages and equal scores beside it."""
    scale = float(torch.tensor(3.0e38))
    gen = torch.Generator().manual_seed(room)
    cache = H.Cache(gen, dtype, 8, 2, 64, 16, [room, 70], [room, 70], scale=scale)
    cache.k[0][torch.isfinite(cache.k[0])] = 0
    _, page, row = cache.slots(0, 0, room)
    cache.k[0, page[137], :, row[137], 0] = 1.0
    cache.table[0, 4:6] = -1
    q = torch.zeros((2, 8, 64), dtype=H.KIND[dtype])
    q[..., 0] = 1.0
    out, lse, weight = run(cache, q, None, torch.zeros_like(cache.weight[0]) if weights else None)
    assert torch.equal(out[0], cache.v[0, page[137], :, row[137]].float().repeat_interleave(4, 0))
    assert float((lse[0].double() / scale - 1).abs().max()) <= 4 * 2.0 ** -24
    for h in range(2):   # all logits of the second sequence are zero
        _, v = cache.rows(cache.v, 1, h, 70)
        assert float((out[1, 4 * h:4 * h + 4].double() - v.mean(0)).abs().max()) <= PAIR * float(v.abs().max())
    assert float((lse[1] - torch.log(torch.tensor(70.0))).abs().max()) <= LOGIT
    if weights:
        assert float(weight[0, :, 137].min()) == float(weight[0, :, 137].max()) == 4 and float(weight[0].sum()) == 8
        assert float((weight[1, :, :70] - 4 / 70).abs().max()) <= 5 * 2.0 ** -24 * 4 / 70
