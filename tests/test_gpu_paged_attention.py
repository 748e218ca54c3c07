"""Attention of one new token over pages, and the weights it accumulates, against float64."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H

pytestmark = pytest.mark.gpu
DEV = H.DEV
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16

# A logit is a sum of head_dim products, in chains of at most 24 roundings: 24 * 2^-24 * sum |q k| * scale, about 10 for these
# inputs, is 1.5e-5 nats.  A weight is off by that relatively, its normalisation again; the log-sum-exp by that absolutely.
LOGIT = 1.5e-5
PAIR = 2 * LOGIT


def run(cache, q, lens, weight=None, lse=True, scratch=0xFF):
    """out, lse, weight of a call whose workspace holds NaN."""
    p = cache.pages
    ws = torch.full((ckv.chunkkv_paged_decode_workspace_bytes(p, weight is not None),), scratch, dtype=torch.uint8, device=DEV)
    out = torch.full((cache.batch, cache.hq, cache.d), float("nan"), device=DEV)
    got = torch.full((cache.batch, cache.hq), float("nan"), device=DEV) if lse else None
    w = None if weight is None else weight.to(DEV)
    n = None if lens is None else torch.as_tensor(lens, dtype=torch.int32).to(DEV)
    ckv.chunkkv_paged_decode_attention(p, cache.table.to(DEV), n, q.to(DEV), cache.pool(cache.k)[0], cache.pool(cache.v)[0], out, got, w, ws)
    return out.cpu(), None if got is None else got.cpu(), None if w is None else w.cpu()


def check(cache, q, lens, with_weights=True):
    want, want_lse, want_weight, top = H.attention(cache, q, lens)
    before = cache.weight[0].clone()
    out, lse, weight = run(cache, q, lens, before if with_weights else None)
    g = cache.hq // cache.hkv
    for b in range(cache.batch):
        for h in range(cache.hkv):
            heads, n = slice(h * g, (h + 1) * g), int(lens[b][h])
            if torch.isinf(want_lse[b, heads]).any():
                assert (out[b, heads] == 0).all() and (lse[b, heads] == float("-inf")).all()
            else:
                assert float((out[b, heads].double() - want[b, heads]).abs().max()) <= PAIR * float(top[b, h])
                assert float((lse[b, heads].double() - want_lse[b, heads]).abs().max()) <= LOGIT
            if with_weights:
                err = (weight[b, h, :n].double() - (before[b, h, :n].double() + want_weight[b, h, :n])).abs()
                # the sum of g weights, then its rounding with what was there
                assert bool((err <= PAIR * want_weight[b, h, :n] + 2.0 ** -24 * (before[b, h, :n].double() + want_weight[b, h, :n])).all())
                assert H.same_bits(weight[b, h, n:], before[b, h, n:])
    return out, lse, weight


SHAPES = [(8, 2, 128), (7, 1, 128), (4, 4, 64), (16, 2, 64), (6, 2, 128), (20, 1, 128)]


@pytest.mark.parametrize("weights", [False, True])
@pytest.mark.parametrize("hq,hkv,d", SHAPES)
@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_short_lengths(lib, dtype, hq, hkv, d, weights):
    """Zero, one, the edges of blocks and steps, in one batch, pages of 16 and of 48 slots."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 48, 63, 65, 127, 128, 129, 160, 200]
    gen = torch.Generator().manual_seed(hq * 100 + d)
    for page, first in ((16, False), (48, True)):
        cache = H.Cache(gen, dtype, hq, hkv, d, page, lens, lens, tokens_first=first)
        check(cache, (torch.randn((len(lens), hq, d), generator=gen)).to(H.KIND[dtype]), cache.len[0].tolist(), weights)


@pytest.mark.parametrize("dtype,hq,hkv,d,page,room", [
    (BF16, 32, 8, 128, 16, [3001]), (F16, 28, 4, 128, 64, [4000, 17, 900, 1]), (BF16, 14, 2, 64, 4096, [9000, 5]), (F32, 8, 2, 128, 32, [2500, 300]),
    (F32, 16, 4, 64, 48, [5000]), (F32, 3, 3, 64, 16, [1500, 1500]), (F16, 12, 1, 128, 256, [20011]), (BF16, 2, 2, 128, 16, [40000]), (F32, 12, 2, 128, 112, [7001]),
])
def test_key_ranges(lib, dtype, hq, hkv, d, page, room):
    """Heads cut into several ranges; lengths that differ between heads, below what there is room for, none."""
    gen = torch.Generator().manual_seed(sum(room))
    cache = H.Cache(gen, dtype, hq, hkv, d, page, room, room)
    q = torch.randn((len(room), hq, d), generator=gen).to(H.KIND[dtype])
    full = [[n] * hkv for n in room]
    for lens in (full, [[max(0, n - 77 * h - 5) for h in range(hkv)] for n in room], [[n // 9 for h in range(hkv)] for n in room], [[0] * hkv for n in room]):
        check(cache, q, lens)
        check(cache, q, lens, False)
    # no lengths: all there is room for; lengths out of range are clamped
    a, b, c = (run(cache, q, x, cache.weight[0]) for x in (None, full, [[n + 1000 for _ in x] for n, x in zip(room, full)]))
    for x, y, z in zip(a, b, c):
        assert H.same_bits(x, y) and H.same_bits(x, z)
    d0 = run(cache, q, [[-5] * hkv for _ in room], None)
    assert (d0[0] == 0).all() and (d0[1] == float("-inf")).all()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 1, 64), (3, 1, 128), (40, 8, 64), (17, 1, 64), (72, 8, 64)])
def test_around_one_workgroup_per_head(lib, dtype, hq, hkv, d):
    """Lengths and numbers of heads at which one workgroup takes a head, of four wavefronts and of eight, or ranges do."""
    gen = torch.Generator().manual_seed(d + hq)
    for batch, top in ((1, 256), (1, 257), (1, 512), (1, 513), (3, 500), (1, 960), (1, 961), (1, 1025), (64 // hkv, 512), (64 // hkv, 513), (128 // hkv, 960), (128 // hkv, 961),
                       (256 // hkv, 40), (264 // hkv, 40)):
        if batch > 32 and d * hq > 700:
            continue
        room = [top if i % 5 == 0 else (i * 37) % top for i in range(batch)]
        cache = H.Cache(gen, dtype, hq, hkv, d, 16, room, room)
        cache.table[0, 3:5] = -1
        check(cache, torch.randn((batch, hq, d), generator=gen).to(H.KIND[dtype]), cache.len[0].tolist())


@pytest.mark.parametrize("dtype", [BF16, F16])
@pytest.mark.parametrize("hq,hkv,d,room", [(16, 1, 128, [45000, 300]), (12, 1, 64, [79000, 1, 4000]), (40, 2, 128, [20600, 0, 33]), (9, 1, 64, [90000])])
@pytest.mark.parametrize("weights", [False, True])
def test_sixteen_heads_at_once(lib, dtype, hq, hkv, d, room, weights):
    """More than eight heads of a kv-head over 20 MB of K and V: one pass over them, in batches of 16."""
    gen = torch.Generator().manual_seed(hq + d)
    cache = H.Cache(gen, dtype, hq, hkv, d, 256, room, [max(0, n - 5) for n in room])
    cache.table[0, 7] = -1
    check(cache, torch.randn((len(room), hq, d), generator=gen).to(H.KIND[dtype]), cache.len[0].tolist(), with_weights=weights)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_many_sequences(lib, dtype):
    """More than a launch's tables hold, most of them short, some empty."""
    gen = torch.Generator().manual_seed(9)
    room = [int(x) for x in torch.randint(0, 150, (150,), generator=gen)]
    room[3], room[131], room[149] = 1300, 2000, 0
    cache = H.Cache(gen, dtype, 4, 2, 64, 16, room, room)
    check(cache, torch.randn((150, 4, 64), generator=gen).to(H.KIND[dtype]), cache.len[0].tolist())


@pytest.mark.parametrize("batch", [1, 15, 16, 17, 33, 127, 128, 129])
def test_sequence_of_a_range(lib, batch):
    gen = torch.Generator().manual_seed(batch)
    room = [1 + (7 * i) % 60 for i in range(batch)]
    room[batch // 2] = 700
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, room, room)
    check(cache, torch.randn((batch, 2, 64), generator=gen).bfloat16(), cache.len[0].tolist())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_pages_that_are_not_there(lib, dtype):
    """Their slots are left out, also when nothing else is left; no entry of a page without slots is used."""
    gen = torch.Generator().manual_seed(4)
    room = [100, 40, 600, 33]
    cache = H.Cache(gen, dtype, 8, 2, 128, 16, room, room)
    cache.table[0, 2] = -1
    cache.table[0, 6] = cache.n_pages
    cache.table[1, :3] = 2 ** 31 - 1
    cache.table[2, 5:30] = -(2 ** 31)
    check(cache, torch.randn((4, 8, 128), generator=gen).to(H.KIND[dtype]), cache.len[0].tolist())


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("scale", [1e-45, 1e-30])
def test_missing_pages_at_vanishing_scales(lib, dtype, scale):
    """Whole steps without a slot that is there, where a scaled mask could vanish too."""
    gen = torch.Generator().manual_seed(14)
    cache = H.Cache(gen, dtype, 4, 1, 64, 16, [900], [900], scale=scale)
    cache.table[0, 2:40] = -1
    check(cache, torch.randn((1, 4, 64), generator=gen).to(H.KIND[dtype]), [[900]])


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("scale", [0.0, 3.0, 1e-30])
def test_scales_and_far_logits(lib, dtype, scale):
    """Logits of some hundred nats: one slot has all the weight; vanishing ones: all have the same."""
    gen = torch.Generator().manual_seed(5)
    cache = H.Cache(gen, dtype, 8, 2, 64, 32, [700, 300], [700, 300], scale=scale)
    q = torch.randn((2, 8, 64), generator=gen).to(H.KIND[dtype])
    if scale == 3.0:
        # the error of a logit grows with the scale: compare where it stays below the bar, on few rows that are far apart
        cache.k[0][torch.isfinite(cache.k[0])] = 0
        s, page, row = cache.slots(0, 0, 700)
        cache.k[0, page[137], :, row[137]] = q[0, 0] / 4
        want, _, _, top = H.attention(cache, q, cache.len[0].tolist())
        out, _, _ = run(cache, q, cache.len[0].tolist())
        assert float((out.double() - want).abs().max()) <= 40 * PAIR * float(top.max())   # sum |q k| * scale up to 4 * 64 * 3 / 2
        return
    check(cache, q, cache.len[0].tolist())


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("room", [200, 400, 3000])
@pytest.mark.parametrize("times", [1.0, 1.2109375])   # a scale times it is exact, or is not
def test_logits_far_below_zero(lib, dtype, room, times):
    """-2^110 / 8 and more for one slot and twice that for the others: it gets all the weight, whatever the softmax starts from."""
    gen = torch.Generator().manual_seed(8)
    cache = H.Cache(gen, dtype, 8, 2, 64, 16, [room], [room])
    there = torch.isfinite(cache.k[0])
    there[..., 1:] = False
    cache.k[0][torch.isfinite(cache.k[0])] = 0
    cache.k[0][there] = -2.0 ** 51
    _, page, row = cache.slots(0, 0, room)
    cache.k[0, page[137], :, row[137], 0] = -2.0 ** 50
    q = torch.zeros((1, 8, 64), dtype=H.KIND[dtype])
    q[..., 0] = times * 2.0 ** 60
    out, lse, weight = run(cache, q, None, torch.zeros_like(cache.weight[0]))
    want = cache.v[0, page[137], :, row[137]].float()
    assert torch.equal(out[0], want.repeat_interleave(4, 0))
    assert float((lse / (-times * 2.0 ** 107) - 1).abs().max()) <= 4 * 2.0 ** -24   # times log2 e, its rounding and back
    assert float(weight[0, :, 137].min()) == float(weight[0, :, 137].max()) == 4 and float(weight[0].sum()) == 8


def test_equal_keys_and_exact_weights(lib):
    """Equal keys: every slot gets g / n, summed over calls."""
    gen = torch.Generator().manual_seed(6)
    cache = H.Cache(gen, BF16, 4, 1, 128, 16, [512], [512])
    cache.k[0][torch.isfinite(cache.k[0])] = 0.5
    q, w = torch.randn((1, 4, 128), generator=gen).bfloat16(), torch.zeros_like(cache.weight[0])
    for i in range(3):
        _, _, w = run(cache, q, [[512]], w)
        assert torch.allclose(w[0, 0, :512], torch.tensor((i + 1) * 4 / 512), rtol=1e-6, atol=0)


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_same_bits_again_and_without_lse(lib, dtype):
    gen = torch.Generator().manual_seed(7)
    cache = H.Cache(gen, dtype, 28, 4, 128, 64, [3000, 5, 1111], [3000, 5, 1111])
    q = torch.randn((3, 28, 128), generator=gen).to(H.KIND[dtype])
    a, b = run(cache, q, None, cache.weight[0]), run(cache, q, None, cache.weight[0], scratch=0)
    for x, y in zip(a, b):
        assert H.same_bits(x, y)
    assert H.same_bits(run(cache, q, None, None, lse=False)[0], run(cache, q, None, None)[0])


def test_refused_by_the_binding(lib):
    gen = torch.Generator().manual_seed(1)
    cache = H.Cache(gen, BF16, 4, 2, 64, 16, [40], [40])
    q, table, n = torch.randn((1, 4, 64), generator=gen).bfloat16().to(DEV), cache.table.to(DEV), cache.len[0].to(DEV)
    kp, out = cache.pool(cache.k)[0], torch.zeros((1, 4, 64), device=DEV)
    ws = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(cache.pages, True), dtype=torch.uint8, device=DEV)
    good = dict(table=table, n=n, q=q, k=kp, v=kp, out=out, lse=None, w=cache.weight[0].to(DEV), ws=ws)
    call = lambda x: ckv.chunkkv_paged_decode_attention(cache.pages, x["table"], x["n"], x["q"], x["k"], x["v"], x["out"], x["lse"], x["w"], x["ws"])  # noqa: E731
    call(good)
    for bad in (dict(table=table[:, :-1]), dict(table=table.long()), dict(n=n[:, :1].contiguous()), dict(q=q.half()), dict(q=q.transpose(1, 2)), dict(k=kp[1:].clone()),
                dict(v=kp.cpu()), dict(out=out.double()), dict(out=out[0, :2]), dict(lse=torch.zeros(3, device=DEV)), dict(w=cache.weight[0]), dict(ws=ws.cpu()), dict(ws=None),
                dict(ws=ws[:-256])):
        with pytest.raises((ValueError, ckv.ChunkKVError)):
            call({**good, **bad})
