"""The calls over pages as a serving loop makes them: compression into pages, then append, attention and eviction step by step; in
graphs, on other streams, over pools past 32-bit offsets, and over long sequences."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from oracle import paged_oracle as orc
from tests import paged_helpers as H
from tests.test_gpu_paged_append import close, turned
from tests.test_gpu_paged_attention import LOGIT, PAIR

pytestmark = pytest.mark.gpu
DEV = H.DEV
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16


@pytest.mark.parametrize("dtype,d,page", [(BF16, 128, 16), (F32, 64, 48), (F16, 128, 64)])
def test_generation_over_a_compressed_prompt(lib, dtype, d, page):
    """Every step's results against float64 from the state before it: rounding does not pile up in the comparison."""
    gen = torch.Generator(device=DEV).manual_seed(d + page)
    hq, hkv, w, c, layers, L = 8, 2, 16, 5, 2, [900, 333]
    kind, B, total = H.KIND[dtype], 2, 1233
    keep = [200, 60]
    prob = ckv.Problem(hq, hkv, d, w, c, dtype, L, keep, [0, 900 * hkv * d], d, hkv * d)
    k, v = ([torch.randn((total, hkv, d), generator=gen, device=DEV).to(kind) for _ in range(layers)] for _ in range(2))
    q_obs = torch.randn((B, hq, w, d), generator=gen, device=DEV).to(kind)
    scores = torch.zeros((B, hkv, prob.score_cap), device=DEV)
    imp = torch.zeros((B, hkv, prob.score_cap * c), device=DEV)
    sel = [torch.zeros((1, B, hkv, prob.sel_cap), dtype=torch.int32, device=DEV) for _ in range(2)]
    cnt = torch.zeros((1, B, hkv), dtype=torch.int32, device=DEV)
    ws = torch.empty(ckv.chunkkv_workspace_bytes(prob, 1, 1), dtype=torch.uint8, device=DEV)
    ckv.chunkkv_score(prob, q_obs, k[0], scores, imp, ws)
    ckv.chunkkv_chunk_topk(prob, scores, *sel, cnt)

    budget = [n + w for n in keep]
    room = [n + 2 for n in budget]
    cache = H.Cache(torch.Generator().manual_seed(1), dtype, hq, hkv, d, page, room, [0, 0], layers=layers)
    table, kp, vp = cache.table.to(DEV), cache.pool(cache.k), cache.pool(cache.v)
    length, pos, weight = cache.len.to(DEV), cache.pos.to(DEV), cache.weight.to(DEV)
    ckv.chunkkv_paged_compact(prob, cache.pages, layers, k, v, *sel, cnt, [imp], table, kp, vp, length, pos, weight)
    for b in range(B):
        for h in range(hkv):
            n = budget[b]
            assert int(length[0, b, h]) == n
            tokens = pos[1, b, h, :n].long()
            assert (tokens.diff() > 0).all() and tokens[-w:].tolist() == list(range(L[b] - w, L[b]))
            assert H.same_bits(weight[0, b, h, :n - w], imp[b, h, tokens[:n - w]]) and (weight[0, b, h, n - w:n] == 0).all()
            rows = (0 if b == 0 else 900) + tokens
            s = torch.arange(n)
            place = (cache.table[b].long()[s // page].to(DEV), h, (s % page).to(DEV))
            assert H.same_bits(kp[1][place], k[1][rows, h]) and H.same_bits(vp[1][place], v[1][rows, h])

    freq = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float()
    qn, kn = ((1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(kind) for _ in range(2))
    ws_a = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(cache.pages, True), dtype=torch.uint8, device=DEV)
    ws_e = torch.empty(ckv.chunkkv_paged_evict_workspace_bytes(cache.pages, layers, budget), dtype=torch.uint8, device=DEV)
    positions = torch.tensor(L, dtype=torch.int32, device=DEV)
    for step in range(6):
        for layer in range(layers):
            qkv = torch.randn((B, hq + 2 * hkv, d), generator=gen, device=DEV).to(kind)
            q_out, before = torch.empty((B, hq, d), dtype=kind, device=DEV), length[layer].clone()
            ckv.chunkkv_paged_append(cache.pages, [1, 1], qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], positions, qn, kn, 1e-6, freq.to(DEV), False, q_out,
                                     table, kp[layer], vp[layer], length[layer], length[layer], pos[layer], weight[layer])
            assert torch.equal(length[layer], before + 1)
            want, size = turned(qkv[:, :hq].cpu(), qn.cpu(), 1e-6, positions.cpu(), freq, False)
            assert close(q_out.cpu(), want, size, dtype)
            out, lse, was = torch.empty((B, hq, d), device=DEV), torch.empty((B, hq), device=DEV), weight[layer].clone()
            ckv.chunkkv_paged_decode_attention(cache.pages, table, length[layer], q_out, kp[layer], vp[layer], out, lse, weight[layer], ws_a)
            cache.k[layer], cache.v[layer] = cache.back([kp[layer]])[0], cache.back([vp[layer]])[0]
            want, want_lse, want_weight, top = H.attention(cache, q_out.cpu(), length[layer].tolist(), layer)
            # logits of rows with norms reach twice the bar's assumption
            assert float((out.cpu().double() - want).abs().max()) <= 2 * PAIR * float(top.max()) and float((lse.cpu().double() - want_lse).abs().max()) <= 2 * LOGIT
            for b in range(B):
                n = int(length[layer, b, 0])
                got, old = weight[layer, b, :, :n].cpu().double(), was[b, :, :n].cpu().double()
                assert bool(((got - old - want_weight[b, :, :n]).abs() <= 2 * PAIR * want_weight[b, :, :n] + 2.0 ** -24 * (old + want_weight[b, :, :n])).all())
                assert int(pos[layer, b, 0, n - 1]) == int(positions[b])
        cache.weight, cache.pos, cache.len = weight.cpu(), pos.cpu(), length.cpu()
        ckv.chunkkv_paged_evict(cache.pages, budget, 8, table, kp, vp, length, pos, weight, ws_e)
        for layer in range(layers):
            for b in range(B):
                for h in range(hkv):
                    n, moves = orc.evict(cache.weight[layer, b, h].numpy(), cache.pos[layer, b, h].numpy(), int(cache.len[layer, b, h]), budget[b], 8)
                    assert n == int(length[layer, b, h]) == budget[b] and len(moves) == 1
                    want = cache.pos[layer, b, h].clone()
                    for source, target in moves:
                        want[target] = cache.pos[layer, b, h, source]
                    assert torch.equal(pos[layer, b, h].cpu(), want)
                    held = set(pos[layer, b, h, :n].tolist())
                    assert set(range(int(positions[b]) - 7, int(positions[b]) + 1)) <= held and len(held) == n
        positions += 1


def loop_state(dtype, seed, room=(300, 77), layers=2, d=128):
    gen = torch.Generator().manual_seed(seed)
    cache = H.Cache(gen, dtype, 8, 2, d, 16, [n + 1 for n in room], list(room), layers=layers)
    cache.pos = torch.where(cache.pos >= 0, cache.pos, -77)
    s = dict(cache=cache, table=cache.table.to(DEV), k=cache.pool(cache.k), v=cache.pool(cache.v), length=cache.len.to(DEV), pos=cache.pos.to(DEV), weight=cache.weight.to(DEV))
    s["qkv"] = torch.randn((layers, 2, 12, d), generator=gen).to(H.KIND[dtype]).to(DEV)
    s["freq"] = (10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64) / d)).float().to(DEV)
    s["positions"] = torch.tensor([5000, 7000], dtype=torch.int32, device=DEV)
    s["q"] = torch.zeros((layers, 2, 8, d), dtype=H.KIND[dtype], device=DEV)
    s["out"], s["lse"] = torch.zeros((layers, 2, 8, d), device=DEV), torch.zeros((layers, 2, 8), device=DEV)
    s["budget"] = list(room)
    s["ws"] = torch.empty(max(ckv.chunkkv_paged_decode_workspace_bytes(cache.pages, True), ckv.chunkkv_paged_evict_workspace_bytes(cache.pages, layers, list(room))),
                          dtype=torch.uint8, device=DEV)
    return s


def step(s, stream=None):
    """One decoding step of every layer; append, attention and eviction share a workspace, one after the other."""
    p = s["cache"].pages
    for layer in range(s["cache"].layers):
        x = s["qkv"][layer]
        ckv.chunkkv_paged_append(p, [1, 1], x[:, :8], x[:, 8:10], x[:, 10:], s["positions"], None, None, 0.0, s["freq"], False, s["q"][layer], s["table"], s["k"][layer],
                                 s["v"][layer], s["length"][layer], s["length"][layer], s["pos"][layer], s["weight"][layer], stream)
        ckv.chunkkv_paged_decode_attention(p, s["table"], s["length"][layer], s["q"][layer], s["k"][layer], s["v"][layer], s["out"][layer], s["lse"][layer], s["weight"][layer],
                                           s["ws"], stream)
    ckv.chunkkv_paged_evict(p, s["budget"], 4, s["table"], s["k"], s["v"], s["length"], s["pos"], s["weight"], s["ws"], stream)
    s["positions"].add_(1)


def same_state(a, b):
    for name in ("length", "pos", "weight", "q", "out", "lse", "positions"):
        assert H.same_bits(a[name], b[name]), name
    for name in ("k", "v"):
        for x, y in zip(a[name], b[name]):
            assert H.same_bits(x, y), name


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_captured_steps(lib, dtype):
    """A captured step replayed against the eager one on a twin state, with eager work and waits between the replays."""
    a, b = loop_state(dtype, 3), loop_state(dtype, 3)
    step(a)
    step(b)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        step(a)
    torch.cuda.synchronize()
    same_state(a, b)                                  # capturing runs nothing
    for i in range(6):
        g.replay()
        torch.cuda.synchronize()
        step(b)
        same_state(a, b)
        if i % 2:
            step(a)
            step(b)
            torch.randn(1 << 20, device=DEV).sum()


def test_two_graphs_share_a_workspace(lib):
    """Attention over two caches through one workspace, captured apart, replayed in turn."""
    s, t = loop_state(BF16, 5), loop_state(BF16, 6)
    t["ws"] = s["ws"]

    def attend(x):
        ckv.chunkkv_paged_decode_attention(x["cache"].pages, x["table"], x["length"][0], x["qkv"][0, :, :8].contiguous(), x["k"][0], x["v"][0], x["out"][0], x["lse"][0], None, x["ws"])

    want = []
    for x in (s, t):
        x["ws"].fill_(0xFF)
        attend(x)
        want.append((x["out"][0].clone(), x["lse"][0].clone()))
    graphs = []
    for x in (s, t):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            attend(x)
        graphs.append(g)
    for i in range(4):
        for x, g, (out, lse) in zip((s, t), graphs, want):
            x["out"].zero_()
            g.replay()
            assert H.same_bits(x["out"][0], out) and H.same_bits(x["lse"][0], lse)


def test_other_streams(lib):
    """A loop on a stream of its own, handed over or current, beside another one on the default stream."""
    a, b, c = (loop_state(F16, 8) for _ in range(3))
    torch.cuda.synchronize()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(3):
        with torch.cuda.stream(s1):
            step(a)
        with torch.cuda.stream(s2):
            step(c, s2)
        step(b)
    torch.cuda.synchronize()
    same_state(a, b)
    same_state(c, b)


def test_shared_pages_are_read_by_both(lib):
    """A common prefix: two sequences whose tables name the same pages."""
    gen = torch.Generator().manual_seed(21)
    cache = H.Cache(gen, BF16, 4, 2, 64, 16, [90, 70], [90, 70])
    cache.table[1, :4] = cache.table[0, :4]
    q = torch.randn((2, 4, 64), generator=gen).bfloat16()
    want, _, _, top = H.attention(cache, q, cache.len[0].tolist())
    out = torch.empty((2, 4, 64), device=DEV)
    ws = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(cache.pages, False), dtype=torch.uint8, device=DEV)
    ckv.chunkkv_paged_decode_attention(cache.pages, cache.table.to(DEV), cache.len[0].to(DEV), q.to(DEV), cache.pool(cache.k)[0], cache.pool(cache.v)[0], out, None, None, ws)
    assert float((out.cpu().double() - want).abs().max()) <= PAIR * float(top.max())


@pytest.mark.parametrize("dtype", [BF16, F32])
def test_offsets_past_32_bits(lib, dtype):
    """Pages at the far end of pools of more than 2^32 bytes and 2^31 elements: append, attention, eviction and compaction there give what
    they give in a small pool."""
    d, hkv, hq, page, room = 128, 2, 4, 64, 200
    kind = H.KIND[dtype]
    pages_far = (1 << 31) // (hkv * page * d) + 8
    gen = torch.Generator(device=DEV).manual_seed(4)
    far_k, far_v = (torch.zeros((pages_far, hkv, page, d), dtype=kind, device=DEV) for _ in range(2))
    near_k, near_v = (torch.zeros((8, hkv, page, d), dtype=kind, device=DEV) for _ in range(2))
    results = []
    for pk, pv, n_pages in ((near_k, near_v, 8), (far_k, far_v, pages_far)):
        gen.manual_seed(4)
        p = ckv.Pages(hq, hkv, d, dtype, page, n_pages, [room])
        table = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2, n_pages - 5]], dtype=torch.int32, device=DEV)
        full = [torch.randn(300 * hkv * d, generator=gen, device=DEV).to(kind) for _ in range(2)]
        prob = ckv.Problem(hq, hkv, d, 16, 10, dtype, [300], [100], [0], 300 * d, d)
        sel = [torch.arange(prob.sel_cap, dtype=torch.int32, device=DEV).repeat(hkv, 1), torch.full((hkv, prob.sel_cap), 10, dtype=torch.int32, device=DEV),
               torch.full((hkv,), 10, dtype=torch.int32, device=DEV)]
        length, pos = torch.zeros((1, hkv), dtype=torch.int32, device=DEV), torch.zeros((1, hkv, room), dtype=torch.int32, device=DEV)
        weight = torch.zeros((1, hkv, room), device=DEV)
        ckv.chunkkv_paged_compact(prob, p, 1, [full[0]], [full[1]], *sel, None, table, [pk], [pv], length, pos, weight)
        qkv = torch.randn((84, hq + 2 * hkv, d), generator=gen, device=DEV).to(kind)
        at = 300 + torch.arange(84, dtype=torch.int32, device=DEV)
        q_out = torch.zeros((84, hq, d), dtype=kind, device=DEV)
        ckv.chunkkv_paged_append(p, [84], qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:], at, None, None, 0.0, None, False, q_out, table, pk, pv, length, length, pos, weight)
        out, lse = torch.zeros((1, hq, d), device=DEV), torch.zeros((1, hq), device=DEV)
        ws = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(p, True), dtype=torch.uint8, device=DEV)
        q = q_out[-1:].contiguous()
        ckv.chunkkv_paged_decode_attention(p, table, length, q, pk, pv, out, lse, weight, ws)
        we = torch.empty(ckv.chunkkv_paged_evict_workspace_bytes(p, 1, [90]), dtype=torch.uint8, device=DEV)
        ckv.chunkkv_paged_evict(p, [90], 20, table, [pk], [pv], length, pos, weight, we)
        results.append([x.clone() for x in (q_out, out, lse, weight, pos, length, pk[table[0].long()], pv[table[0].long()])])
    for x, y in zip(*results):
        assert H.same_bits(x, y)
    assert int(results[0][5][0, 0]) == 90 and float(results[0][1].abs().max()) > 0


@pytest.mark.parametrize("dtype,page,n", [(BF16, 48, 1_300_003), (F32, 16, 500_001)])
def test_long_sequences(lib, dtype, page, n):
    """More than a thousand ranges and blocks past 2^16, an odd number of blocks per page; eviction of the same cache."""
    gen = torch.Generator(device=DEV).manual_seed(n)
    d, hq, kind, held = 64, 2, H.KIND[dtype], -(-n // page)
    k, v = (torch.randn((held, 1, page, d), generator=gen, device=DEV).to(kind) for _ in range(2))
    table = torch.randperm(held, generator=gen, device=DEV).to(torch.int32)[None]
    q = torch.randn((1, hq, d), generator=gen, device=DEV).to(kind)
    p = ckv.Pages(hq, 1, d, dtype, page, held, [n])
    out, lse, weight = torch.zeros((1, hq, d), device=DEV), torch.zeros((1, hq), device=DEV), torch.zeros((1, 1, n), device=DEV)
    ws = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(p, True), dtype=torch.uint8, device=DEV)
    ckv.chunkkv_paged_decode_attention(p, table, None, q, k, v, out, lse, weight, ws)
    kk, vv = (x[table[0].long(), 0].reshape(-1, d)[:n].double() for x in (k, v))
    x = torch.mm(q[0].double(), kk.t().contiguous()) * d ** -0.5
    want_lse = torch.logsumexp(x, 1)
    w = torch.exp(x - want_lse[:, None])
    # the sums over a million slots add their own roundings: 2^-24 for each level of threads, wavefronts and ranges, some 60 in a chain
    assert float((lse[0].double() - want_lse).abs().max()) <= LOGIT + 60 * 2.0 ** -24
    assert float((out[0].double() - torch.mm(w, vv)).abs().max()) <= (PAIR + 120 * 2.0 ** -24) * float(vv.abs().max())
    assert bool(((weight[0, 0].double() - w.sum(0)).abs() <= (PAIR + 120 * 2.0 ** -24) * w.sum(0)).all())
    budget, recent = n - 20_000, 1000
    pos = torch.randperm(n, generator=gen, device=DEV).to(torch.int32)[None, None]
    length, before, was = torch.full((1, 1), n, dtype=torch.int32, device=DEV), weight.clone(), pos.clone()
    we = torch.empty(ckv.chunkkv_paged_evict_workspace_bytes(p, 1, [budget]), dtype=torch.uint8, device=DEV)
    old_k = k.clone()
    ckv.chunkkv_paged_evict(p, [budget], recent, table, [k], [v], length, pos, weight, we)
    key = torch.where(was[0, 0] > int(was.max()) - recent, float("inf"), before[0, 0])
    kept = torch.sort(key, descending=True, stable=True).indices[:budget].sort().values
    stays = torch.zeros(n, dtype=torch.bool, device=DEV)
    stays[kept] = True
    to, source = (~stays[:budget]).nonzero()[:, 0], kept[kept >= budget]
    want = was[0, 0].clone()
    want[to] = was[0, 0][source]
    assert int(length) == budget and torch.equal(pos[0, 0], want)
    place = lambda s: (table[0].long()[s // page], 0, s % page)  # noqa: E731
    assert H.same_bits(k[place(to)], old_k[place(source)]) and H.same_bits(k[place(kept[kept < budget])], old_k[place(kept[kept < budget])])
