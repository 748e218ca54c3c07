"""The gather into pages for selections that cut more than one chunk, for counts and chunk sizes of any size: bit for bit."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H

pytestmark = pytest.mark.gpu
DEV = H.DEV
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16


def cut_chunks(gen, P, c, n_keep, entries):
    """Ascending chunks and lengths of so many entries, n_keep tokens in all, most of the chunks cut."""
    pick = torch.randperm(-(-P // c), generator=gen)[:entries].sort().values
    room = torch.clamp(P - pick * c, max=c)
    size = torch.ones(entries, dtype=torch.long)
    while int(size.sum()) < n_keep:
        i = int(torch.randint(0, entries, (1,), generator=gen))
        size[i] += int(size[i] < room[i])
    return pick, size


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("dtype,d,L,keep,c,cap,entries,layers,reuse", [
    (BF16, 128, [200, 90], [64, 0], 8, 40, 20, 3, 2), (F16, 64, [3000], [100], 10, 300, 100, 1, 1), (F32, 64, [5000, 40], [130, 5], 300, 17, 5, 2, 1),
    (BF16, 64, [9000] + [60] * 17, [1700] + [9] * 17, 5, 1700, 900, 2, 2), (F32, 128, [20000], [2500], 7, 2600, 2400, 1, 1),
])
def test_many_cut_chunks(lib, dtype, d, L, keep, c, cap, entries, layers, reuse, whole):
    """What the selection's rules allow and the library's own never does: more entries than ceil(n_keep / c) + 1."""
    gen = torch.Generator().manual_seed(sum(L) + c)
    w, B, hkv, groups, kind = 16, len(L), 2, -(-layers // reuse), H.KIND[dtype]
    bases = [sum(L[:b]) * hkv * d for b in range(B)]
    prob = ckv.Problem(4, hkv, d, w, c, dtype, L, keep, bases, d, hkv * d, sel_cap=cap, flags=ckv.FLAG_WHOLE_CHUNKS if whole else 0)
    full = [[torch.randn(sum(L) * hkv * d, generator=gen).to(kind) for _ in range(layers)] for _ in range(2)]
    sel = [torch.full((groups, B, hkv, cap), -5, dtype=torch.int32) for _ in range(2)] + [torch.zeros((groups, B, hkv), dtype=torch.int32)]
    picks = {}
    for g in range(groups):
        for b in range(B):
            for h in range(hkv):
                n = min(entries + h if entries + h <= keep[b] else keep[b], -(-(L[b] - w) // c))
                pick, size = cut_chunks(gen, L[b] - w, c, keep[b], n) if n else (torch.zeros(0, dtype=torch.long),) * 2
                sel[0][g, b, h, :n], sel[1][g, b, h, :n], sel[2][g, b, h] = pick.int(), size.int(), n
                picks[g, b, h] = [int(p) * c + i for p, s in zip(pick, size) for i in range(int(s))] + list(range(L[b] - w, L[b]))
    cache = H.Cache(gen, dtype, 4, hkv, d, 16, [n + w for n in keep], [0] * B, layers=layers)
    want = [x.clone() for x in (cache.k, cache.v, cache.pos, cache.weight, cache.len)]
    for layer in range(layers):
        for b in range(B):
            for h in range(hkv):
                tokens = torch.tensor(picks[layer // reuse, b, h])
                n = len(tokens)
                assert n == keep[b] + w
                want[4][layer, b, h] = n
                want[2][layer, b, h, :n], want[3][layer, b, h, :n] = tokens.int(), 0.0
                s = torch.arange(n)
                place = (layer, cache.table[b].long()[s // 16], h, s % 16)
                rows = bases[b] + h * d + tokens[:, None] * hkv * d + torch.arange(d)
                want[0][place], want[1][place] = full[0][layer][rows], full[1][layer][rows]
    kp, vp = cache.pool(cache.k), cache.pool(cache.v)
    length, pos, weight = cache.len.to(DEV), cache.pos.to(DEV), cache.weight.to(DEV)
    up = lambda xs: [x.to(DEV) for x in xs]  # noqa: E731
    ckv.chunkkv_paged_compact(prob, cache.pages, reuse, up(full[0]), up(full[1]), *up(sel), None, cache.table.to(DEV), kp, vp, length, pos, weight)
    for name, x, y in zip(("k", "v", "pos", "weight", "length"), (cache.back(kp), cache.back(vp), pos.cpu(), weight.cpu(), length.cpu()), want):
        assert H.same_bits(x, y), name


@pytest.mark.parametrize("whole", [False, True])
@pytest.mark.parametrize("cap,count", [(9, 10 ** 6), (200, 200), (5000, 10 ** 6), (200, -1)])
def test_counts_out_of_bounds(lib, cap, count, whole):
    """Whatever a count says: the window is stored behind the kept rows, the length is written."""
    gen = torch.Generator().manual_seed(cap)
    prob = ckv.Problem(2, 1, 64, 16, 8, BF16, [200], [64], [0], 200 * 64, 64, sel_cap=cap, flags=ckv.FLAG_WHOLE_CHUNKS if whole else 0)
    k, v = (torch.randn(200 * 64, generator=gen).bfloat16() for _ in range(2))
    # the first chunk over and over: eight rows an entry until the budget is full, and no row of any entry behind
    sel = [torch.zeros(cap, dtype=torch.int32, device=DEV), torch.full((cap,), 8, dtype=torch.int32, device=DEV), torch.tensor([count], dtype=torch.int32, device=DEV)]
    kept = 64 if count > 0 else (0 if whole else None)
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, [80], [0])
    kp, vp, n, pos = cache.pool(cache.k), cache.pool(cache.v), cache.len.to(DEV), cache.pos.to(DEV)
    ckv.chunkkv_paged_compact(prob, cache.pages, 1, [k.to(DEV)], [v.to(DEV)], *sel, None, cache.table.to(DEV), kp, vp, n, pos, None)
    at = 64 if kept is None else kept
    tokens = ([] if kept is None else list(range(8)) * (kept // 8)) + list(range(184, 200))
    assert int(n) == at + 16
    s = torch.arange(at + 16 - len(tokens), at + 16)
    place = (0, cache.table[0].long()[s // 16], 0, s % 16)
    want_k, want_v, want_pos = cache.k.clone(), cache.v.clone(), cache.pos.clone()
    want_k[place], want_v[place] = k.view(200, 64)[tokens], v.view(200, 64)[tokens]
    want_pos[0, 0, 0, s] = torch.tensor(tokens, dtype=torch.int32)
    assert H.same_bits(cache.back(kp), want_k) and H.same_bits(cache.back(vp), want_v) and H.same_bits(pos.cpu(), want_pos)


@pytest.mark.parametrize("c", [2 ** 24 + 1, 2 ** 31 - 20, 2 ** 31 - 1])
def test_chunks_longer_than_any_prefix(lib, c):
    """One chunk holds the whole prefix, whatever its size is said to be."""
    gen = torch.Generator().manual_seed(5)
    k, v = (torch.randn(200 * 64, generator=gen).bfloat16() for _ in range(2))
    prob = ckv.Problem(2, 1, 64, 16, c, BF16, [200], [64], [0], 200 * 64, 64)
    sel = [torch.tensor(x, dtype=torch.int32, device=DEV) for x in ([0, -1], [64, -1], [1])]
    cache = H.Cache(gen, BF16, 2, 1, 64, 16, [80], [0])
    kp, vp, n, pos = cache.pool(cache.k), cache.pool(cache.v), cache.len.to(DEV), cache.pos.to(DEV)
    ckv.chunkkv_paged_compact(prob, cache.pages, 1, [k.to(DEV)], [v.to(DEV)], *sel, None, cache.table.to(DEV), kp, vp, n, pos, None)
    tokens, s = list(range(64)) + list(range(184, 200)), torch.arange(80)
    want_k, want_v = cache.k.clone(), cache.v.clone()
    place = (0, cache.table[0].long()[s // 16], 0, s % 16)
    want_k[place], want_v[place] = k.view(200, 64)[tokens], v.view(200, 64)[tokens]
    assert int(n) == 80 and pos[0, 0, 0, :80].tolist() == tokens
    assert H.same_bits(cache.back(kp), want_k) and H.same_bits(cache.back(vp), want_v)
