"""Eviction by accumulated weight, in place, and the gather of a selection into pages: bit for bit against the oracle."""
import numpy as np
import pytest
import torch

import paper_2502_00299_amd as ckv
from oracle import paged_oracle as orc
from tests import paged_helpers as H

pytestmark = pytest.mark.gpu
DEV = H.DEV
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16


def evicted(cache, budget, recent):
    """The arrays after the eviction, by the oracle's moves."""
    k, v, length, pos, weight = cache.k.clone(), cache.v.clone(), cache.len.clone(), cache.pos.clone(), cache.weight.clone()
    for layer in range(cache.layers):
        for b in range(cache.batch):
            for h in range(cache.hkv):
                n, moves = orc.evict(cache.weight[layer, b, h].numpy(), cache.pos[layer, b, h].numpy(), int(length[layer, b, h]), budget[b], recent)
                for source, target in moves:
                    pos[layer, b, h, target], weight[layer, b, h, target] = pos[layer, b, h, source], weight[layer, b, h, source]
                    place = [(int(cache.table[b, s // cache.page]), h, s % cache.page) for s in (source, target)]
                    if all(0 <= p[0] < cache.n_pages for p in place):
                        k[(layer, *place[1])], v[(layer, *place[1])] = cache.k[(layer, *place[0])], cache.v[(layer, *place[0])]
                length[layer, b, h] = n
    return k, v, length, pos, weight


def check(cache, budget, recent):
    want = evicted(cache, budget, recent)
    kp, vp = cache.pool(cache.k), cache.pool(cache.v)
    length, pos, weight = cache.len.to(DEV), cache.pos.to(DEV), cache.weight.to(DEV)
    ws = torch.full((ckv.chunkkv_paged_evict_workspace_bytes(cache.pages, cache.layers, budget),), 0xFF, dtype=torch.uint8, device=DEV)
    ckv.chunkkv_paged_evict(cache.pages, budget, recent, cache.table.to(DEV), kp, vp, length, pos, weight, ws)
    got = (cache.back(kp), cache.back(vp), length.cpu(), pos.cpu(), weight.cpu())
    for name, x, y in zip(("k", "v", "length", "pos", "weight"), got, want):
        assert H.same_bits(x, y), name


@pytest.mark.parametrize("dtype,d", [(BF16, 128), (F16, 64), (F32, 128), (F32, 64)])
@pytest.mark.parametrize("room,budget,recent", [
    ([33], [32], 0), ([33], [32], 32), ([200, 64, 5, 1], [50, 64, 5, 1], 1), ([300, 17, 0], [20, 3, 0], 0), ([260, 255], [130, 254], 16), ([1000, 30], [1, 29], 1),
    ([40], [0], 0), ([1500], [700], 64), ([40, 40], [41, 39], 20),
])
def test_against_the_oracle(lib, dtype, d, room, budget, recent):
    gen = torch.Generator().manual_seed(sum(room) + recent)
    for page, first, layers in ((16, False, 2), (48, True, 1)):
        cache = H.Cache(gen, dtype, 4, 2, d, page, room, room, layers=layers, tokens_first=first)
        cache.len[:, :, 1] -= (cache.len[:, :, 1] > 3).int() * 2         # heads of different length
        check(cache, budget, recent)


@pytest.mark.parametrize("n,budget", [(256, 100), (257, 256), (1024, 1000), (1025, 3), (4096, 2000), (4097, 4096), (16384, 16000), (16385, 9000), (40000, 39000)])
def test_lengths_at_which_the_selection_changes(lib, n, budget):
    gen = torch.Generator().manual_seed(n)
    cache = H.Cache(gen, BF16, 2, 1, 64, 64, [n], [n])
    cache.weight[0, 0, 0, :n] = torch.randn(n, generator=gen).mul(2).exp()
    check(cache, [budget], min(100, budget))


@pytest.mark.parametrize("kind", ["equal", "two values", "zeros", "negative zero", "infinite", "tiny"])
def test_ties_and_odd_weights(lib, kind):
    gen = torch.Generator().manual_seed(11)
    cache = H.Cache(gen, F16, 2, 2, 64, 16, [700], [700])
    w = cache.weight[0, 0, :, :700]
    if kind == "equal":
        w[:] = 3.25
    elif kind == "two values":
        w[:] = (torch.rand(w.shape, generator=gen) < 0.5).float()
    elif kind == "zeros":
        w[:] = 0.0
    elif kind == "negative zero":
        w[:] = torch.where(torch.rand(w.shape, generator=gen) < 0.5, 0.0, -0.0)
    elif kind == "infinite":
        w[torch.rand(w.shape, generator=gen) < 0.6] = float("inf")
    else:
        w *= 1e-40
    for recent in (0, 7):
        check(cache, [333], recent)


def test_equal_positions_and_their_ends(lib):
    """All positions alike: all protected, the lower slots stay; positions at both ends of the type."""
    gen = torch.Generator().manual_seed(12)
    cache = H.Cache(gen, BF16, 1, 1, 64, 16, [100], [100])
    cache.pos[0, 0, 0, :100] = 5
    check(cache, [30], 3)
    cache.pos[0, 0, 0, :100] = torch.randint(-(2 ** 31), 2 ** 31 - 1, (100,), generator=gen).to(torch.int32)
    cache.pos[0, 0, 0, 17], cache.pos[0, 0, 0, 18] = 2 ** 31 - 1, -(2 ** 31)
    check(cache, [30], 30)
    cache.pos[0, 0, 0, :100] = -(2 ** 31) + torch.arange(100, dtype=torch.int32)
    check(cache, [30], 30)


def test_many_layers_and_sequences(lib):
    gen = torch.Generator().manual_seed(13)
    room = [20 + i % 9 for i in range(131)]
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, room, room, layers=35)
    check(cache, [n - 3 for n in room], 2)


def test_pages_that_are_not_there(lib):
    gen = torch.Generator().manual_seed(14)
    cache = H.Cache(gen, BF16, 2, 2, 64, 16, [90], [90])
    cache.table[0, 1], cache.table[0, 5] = -4, cache.n_pages
    check(cache, [45], 5)


# ---- gather into pages ------------------------------------------------------------------------------------------------


def selection(gen, P, c, n_keep, whole):
    """Chunks and lengths of one head, as the library's selection makes them."""
    C = -(-P // c)
    m = min(n_keep // c, C) if whole else -(-n_keep // c)
    pick = torch.randperm(C, generator=gen)[:m].sort().values
    size = torch.clamp(P - pick * c, max=c)
    if whole:
        return pick, size
    while int(size.sum()) < n_keep:      # the ragged last chunk is short: one more
        pick = torch.tensor(sorted(set(pick.tolist()) | {next(i for i in range(C) if i not in set(pick.tolist()))}))
        size = torch.clamp(P - pick * c, max=c)
    over = int(size.sum()) - n_keep
    cut = next(i for i in range(len(size)) if int(size[i]) > over) if over else 0
    size[cut] -= over
    return pick, size


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("dtype,d,hkv,L,keep,c,layers,reuse,packed", [
    (BF16, 128, 2, [500], [100], 10, 3, 2, False), (F16, 64, 3, [700, 33, 40], [301, 0, 7], 5, 2, 1, True), (F32, 128, 1, [400], [200], 1, 1, 1, False),
    (F32, 64, 2, [1000, 900], [333, 100], 300, 2, 2, True), (BF16, 64, 1, [32, 45], [0, 13], 20, 1, 1, True), (BF16, 128, 4, [3000], [2968], 3, 2, 3, False),
    (F16, 128, 2, [5000] + [100] * 18, [900] + [20] * 18, 33, 33, 5, True),
])
def test_compact_into_pages(lib, dtype, d, hkv, L, keep, c, layers, reuse, packed, whole):
    gen = torch.Generator().manual_seed(sum(L) + c)
    w, B, hq, groups = 32, len(L), 2 * hkv, -(-layers // reuse)
    kind = H.KIND[dtype]
    bases, total = [sum(L[:b]) * hkv * d for b in range(B)], sum(L)
    strides = (d, hkv * d) if packed or B > 1 else (L[0] * d, d)
    prob = ckv.Problem(hq, hkv, d, w, c, dtype, L, keep, bases, *strides, flags=ckv.FLAG_WHOLE_CHUNKS if whole else 0)
    full = [[torch.randn(total * hkv * d, generator=gen).to(kind) for _ in range(layers)] for _ in range(2)]
    sel = torch.full((groups, B, hkv, prob.sel_cap), -5, dtype=torch.int32), torch.full((groups, B, hkv, prob.sel_cap), -5, dtype=torch.int32), torch.zeros((groups, B, hkv), dtype=torch.int32)
    picks = {}
    for g in range(groups):
        for b in range(B):
            for h in range(hkv):
                pick, size = selection(gen, L[b] - w, c, keep[b], whole) if keep[b] else (torch.zeros(0, dtype=torch.long),) * 2
                sel[0][g, b, h, :len(pick)], sel[1][g, b, h, :len(pick)], sel[2][g, b, h] = pick.int(), size.int(), len(pick)
                picks[g, b, h] = [int(p) * c + i for p, s in zip(pick, size) for i in range(int(s))] + list(range(L[b] - w, L[b]))
    imp = [torch.rand((B, hkv, prob.score_cap * c), generator=gen) for _ in range(groups)]
    room = [n + w for n in keep]
    cache = H.Cache(gen, dtype, hq, hkv, d, 16, room, [0] * B, layers=layers, tokens_first=packed)
    for with_weights in (True, False):
        want = [x.clone() for x in (cache.k, cache.v, cache.pos, cache.weight, cache.len)]
        for layer in range(layers):
            for b in range(B):
                for h in range(hkv):
                    tokens = picks[layer // reuse, b, h]
                    n = len(tokens)
                    want[4][layer, b, h] = n
                    want[2][layer, b, h, :n] = torch.tensor(tokens, dtype=torch.int32)
                    want[3][layer, b, h, :n] = 0.0
                    if with_weights:
                        want[3][layer, b, h, :n - w] = imp[layer // reuse][b, h, tokens[:n - w]]
                    s = torch.arange(n)
                    page, row = cache.table[b].long()[s // 16], s % 16
                    rows = bases[b] + h * strides[0] + torch.tensor(tokens)[:, None] * strides[1] + torch.arange(d)
                    want[0][layer, page, h, row], want[1][layer, page, h, row] = full[0][layer][rows], full[1][layer][rows]
        kp, vp = cache.pool(cache.k), cache.pool(cache.v)
        length, pos, weight = cache.len.to(DEV), cache.pos.to(DEV), cache.weight.to(DEV)
        ckv.chunkkv_paged_compact(prob, cache.pages, reuse, [x.to(DEV) for x in full[0]], [x.to(DEV) for x in full[1]], *[x.to(DEV) for x in sel],
                                  [x.to(DEV) for x in imp] if with_weights else None, cache.table.to(DEV), kp, vp, length, pos, weight)
        for name, x, y in zip(("k", "v", "pos", "weight", "length"), (cache.back(kp), cache.back(vp), pos.cpu(), weight.cpu(), length.cpu()), want):
            assert H.same_bits(x, y), name
    # without positions and weights the rows are the same
    kp2, vp2 = cache.pool(cache.k), cache.pool(cache.v)
    ckv.chunkkv_paged_compact(prob, cache.pages, reuse, [x.to(DEV) for x in full[0]], [x.to(DEV) for x in full[1]], *[x.to(DEV) for x in sel], None, cache.table.to(DEV),
                              kp2, vp2, length, None, None)
    assert H.same_bits(cache.back(kp2), want[0]) and H.same_bits(cache.back(vp2), want[1])


def test_malformed_selections_store_nothing(lib):
    """Entries that are out of bounds are skipped: nothing outside a head's slots and the full cache is touched."""
    gen = torch.Generator().manual_seed(1)
    prob = ckv.Problem(2, 1, 64, 16, 8, BF16, [200], [64], [0], 200 * 64, 64)
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, [80], [0])
    k = torch.randn(200 * 64, generator=gen).bfloat16().to(DEV)
    cap = prob.sel_cap
    for chunk, length, count in (([-1] * cap, [8] * cap, cap), ([5000] * cap, [8] * cap, cap), ([3] * cap, [9] * cap, 8), ([3] * cap, [0] * cap, 8), ([22] * cap, [8] * cap, 4),
                                 ([0] * cap, [8] * cap, 10 ** 6), ([0] * cap, [8] * cap, -3), ([0] * cap, [2 ** 31 - 1] * cap, 8)):
        sel = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in (chunk, length, [count])]
        kp, vp = cache.pool(cache.k), cache.pool(cache.v)
        n, pos = cache.len.to(DEV), cache.pos.to(DEV)
        ckv.chunkkv_paged_compact(prob, cache.pages, 1, [k], [k], *sel, None, cache.table.to(DEV), kp, vp, n, pos, None)
        used = cache.table[0, :5].long()
        got, kept = cache.back(kp), cache.k.clone()
        kept[0, used] = got[0, used]
        assert H.same_bits(got, kept) and (n == 80).all() and H.same_bits(pos.cpu()[..., 80:], cache.pos[..., 80:])


def test_refused_by_the_binding(lib):
    gen = torch.Generator().manual_seed(1)
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, [80], [80])
    kp, vp, n, pos, w = cache.pool(cache.k), cache.pool(cache.v), cache.len.to(DEV), cache.pos.to(DEV), cache.weight.to(DEV)
    ws = torch.empty(ckv.chunkkv_paged_evict_workspace_bytes(cache.pages, 1, [70]), dtype=torch.uint8, device=DEV)
    good = dict(budget=[70], recent=3, table=cache.table.to(DEV), k=kp, v=vp, n=n, pos=pos, w=w, ws=ws)
    call = lambda x: ckv.chunkkv_paged_evict(cache.pages, x["budget"], x["recent"], x["table"], x["k"], x["v"], x["n"], x["pos"], x["w"], x["ws"])  # noqa: E731
    for bad in (dict(budget=[70, 1]), dict(recent=71), dict(recent=-1), dict(k=[kp[0][:-1].clone()]), dict(v=[]), dict(v=[vp[0].float()]), dict(n=n.cpu()), dict(pos=pos[..., :-1].contiguous()),
                dict(w=w.double()), dict(ws=ws.cpu()), dict(ws=None), dict(ws=ws[:-1])):
        with pytest.raises((ValueError, ckv.ChunkKVError)):
            call({**good, **bad})
    call(good)
    prob = ckv.Problem(2, 1, 64, 16, 8, BF16, [200], [64], [0], 200 * 64, 64)
    sel = [torch.zeros(prob.sel_cap, dtype=torch.int32, device=DEV) for _ in range(2)] + [torch.zeros(1, dtype=torch.int32, device=DEV)]
    full = torch.zeros(200 * 64, dtype=torch.bfloat16, device=DEV)
    fill = lambda x: ckv.chunkkv_paged_compact(prob, cache.pages, 1, x["k"], x["v"], *x["sel"], x["imp"], good["table"], x["kp"], vp, x["n"], pos, None)  # noqa: E731
    good = {**good, "k": [full], "v": [full], "sel": sel, "imp": None, "kp": kp}
    fill(good)
    for bad in (dict(k=[full[:-1].clone()]), dict(v=[full.cpu()]), dict(v=[full, full]), dict(k=[full.half()]), dict(sel=[sel[0], sel[1][1:], sel[2]]), dict(kp=[kp[0][1:].clone()]),
                dict(imp=[]), dict(imp=[torch.zeros(100, device=DEV)]), dict(n=n.long())):
        with pytest.raises((ValueError, ckv.ChunkKVError)):
            fill({**good, **bad})
