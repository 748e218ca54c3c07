"""Operators of a serving loop over a paged cache, as cases that can be timed and compared.

A prompt's cache has been compressed; from then on every step puts the new token's key and value into pages, attends over
them, and keeps the cache at its budget.  Four operators: the gather of a selection into pages (`compact`), the new
tokens' head norms, rotation and storing (`append`), the attention of one new token with the accumulation of its weights
(`attend`), and the eviction by those weights (`evict`).

Keys and queries have the structure of the repository's generator: N(0,1) and a shared direction whose strength is
graded over runs of tokens (about 2 nats of the logit), so attention is uneven as over a prompt.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}

# Eight prompts of 4096 to 65536 tokens, uniformly drawn: the repository's ragged batch.
RAGGED = "54883 20995 52241 22450 47422 10460 26034 41231"
# A full serving batch: 64 sequences between 500 and 8000 tokens.
SERVED = " ".join(str(500 + (i * 4733) % 7501) for i in range(64))


def _case(name, mode, lens, **kw):
    case = dict(name=name, mode=mode, lens=lens, new="1", layers=1, q_heads=32, kv_heads=8, dim=128, dtype="bf16", page=64, tokens_first=False,
                uneven=False, weights=False, norm=True, rotary=128, interleaved=False, window=32, chunk=10, keep=10, reuse=1, budget=0, recent=32)
    case.update(kw)
    return case


def listed():
    return [
        # a decoding step of eight sequences, one layer
        _case("append_step_b8", "append", "848 900 1000 1300 848 848 2000 860"),
        # a chunk of a prompt beside single tokens of other sequences, fp16, half of the head rotated in neighbouring pairs, no norms
        _case("append_mixed_f16", "append", "0 4000 801 17 12000", new="1777 1 1 300 1", q_heads=28, kv_heads=4, dtype="f16", page=16, norm=False,
              rotary=64, interleaved=True),
        # a whole 8K prompt
        _case("append_prompt_8k", "append", "0", new="8192"),
        # one layer's attention of a decoding step over an 8K prompt kept at 10 %
        _case("attend_8k_kept", "attend", "848", page=16, weights=True),
        # fp32 caches, ragged, heads of unequal length
        _case("attend_f32_d64", "attend", "3111 8000 75 1", q_heads=16, kv_heads=4, dim=64, dtype="f32", page=48, uneven=True, weights=True),
        # a full batch of sequences, fp16, tokens of all heads together in a page
        _case("attend_b64_f16", "attend", SERVED, q_heads=28, kv_heads=4, dtype="f16", page=32, tokens_first=True),
        # a 128K prompt with its full cache, accumulating weights
        _case("attend_128k", "attend", "131072", page=128, weights=True),
        # the ragged batch over its full caches
        _case("attend_ragged", "attend", RAGGED, q_heads=28, kv_heads=4, page=256),
        # one layer of an 8K prompt at 10 % into pages
        _case("compact_8k", "compact", "8192", weights=True, page=16),
        # a 32K prompt at 20 %, all layers, two per selection
        _case("compact_32k_stack", "compact", "32768", layers=32, keep=20, reuse=2, page=64),
        # a generated token too many in every layer: one slot leaves
        _case("evict_step", "evict", "849", layers=32, budget=848, page=16),
        # half of the cache leaves four sequences in eight layers
        _case("evict_half", "evict", "16384 12000 9000 16001", layers=8, q_heads=28, kv_heads=4, budget=8192, recent=256, page=64),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    mode = rng.choice(["append", "append", "attend", "attend", "attend", "compact", "evict"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (28, 4), (16, 4), (8, 8), (4, 2), (64, 8)])
    dim = rng.choice([128, 128, 64])
    page = rng.choice([16, 16, 32, 48, 64, 128, 256])
    batch = rng.choice([1, 1, 2, 5, 8, 17, 64])
    case = dict(mode=mode, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, page=page, tokens_first=rng.random() < 0.3)
    row = kv_heads * dim
    if mode == "append":
        new = [_log_uniform(rng, 1, 8192 / batch) if rng.random() < 0.6 else 1 for _ in range(batch)]
        while sum(new) * (q_heads + 2 * kv_heads) * dim > (5e7 if dtype != "f32" else 2.5e7):
            new = [max(1, n // 2) for n in new]
        lens = [rng.choice([0, _log_uniform(rng, 1, 3000)]) for _ in range(batch)]
        case.update(_rest(lens, new="%s" % " ".join(map(str, new)), norm=rng.random() < 0.6, rotary=rng.choice([dim, dim, dim // 2, 16, 0]),
                          interleaved=rng.random() < 0.4, weights=rng.random() < 0.5, uneven=rng.random() < 0.3))
        return case
    top = _log_uniform(rng, 1 if mode == "attend" else 200, 131072)
    lens = [top] + [max(1, int(top * rng.uniform(0.05, 1.0))) for _ in range(batch - 1)]
    if mode == "attend":
        while batch * max(lens) * row > (2.5e8 if dtype != "f32" else 6e7) or sum(lens) * row > 1.4e8:
            lens = [max(1, n // 2) for n in lens]
        case.update(_rest(lens, uneven=rng.random() < 0.3, weights=rng.random() < 0.5))
        return case
    window = rng.choice([16, 32])
    while sum(lens) * row > 1.3e8:
        lens = [n // 2 for n in lens]
    chunk = rng.choice([1, 3, 5, 10, 20, 33])
    lens = [max(window + 4 * chunk, n) for n in lens]
    layers = max(1, min(rng.choice([1, 2, 7, 16, 32]), int((8e8 if mode == "compact" else 2e8) / (sum(lens) * row * (2 if dtype == "f32" else 1)))))
    if mode == "compact":
        case.update(_rest(lens, layers=layers, window=window, chunk=chunk, keep=rng.choice([5, 10, 20, 30]),
                          reuse=rng.choice([1, 2, 3]), weights=rng.random() < 0.5))
    else:
        least = min(lens)
        budget = rng.choice([least - 1, least - rng.randint(1, least // 2), max(8, int(max(lens) * rng.uniform(0.2, 0.9)))])
        case.update(_rest(lens, layers=layers, budget=budget, recent=rng.choice([0, 1, min(32, budget), budget // 4]), weights=True))
    return case


def _rest(lens, **kw):
    case = _case("", "", " ".join(map(str, lens)))
    case.update(kw)
    return {k: case[k] for k in ("lens", "new", "layers", "uneven", "weights", "norm", "rotary", "interleaved", "window", "chunk", "keep", "reuse", "budget", "recent")}


def _ints(text):
    return [int(x) for x in text.split()]


# ---- inputs -------------------------------------------------------------------------------------------------------


class _State:
    pass


def _capacity(case):
    """Slots that every sequence has room for."""
    lens, new = _ints(case["lens"]), _ints(case["new"])
    if case["mode"] == "append":
        return [n + new[i % len(new)] for i, n in enumerate(lens)]
    if case["mode"] == "compact":
        return [case["keep"] * (n - case["window"]) // 100 + case["window"] for n in lens]
    return lens


def _strength(d):
    return math.sqrt(2.0 * math.sqrt(d))


def _pages(s, gen, u):
    """The pools of all layers, [layers][pages][kv_heads][page][dim] or with the tokens before the heads: what earlier steps
    left in them, rows past a sequence's last one too."""
    c = s.case
    h, d, pt, kind = c["kv_heads"], c["dim"], c["page"], DTYPE[c["dtype"]]
    shape = (c["layers"], s.n_pages, pt, h, d) if c["tokens_first"] else (c["layers"], s.n_pages, h, pt, d)
    k, v = (torch.empty(shape, dtype=kind, device=DEV).normal_(generator=gen) for _ in range(2))
    if u is not None:
        level = torch.randn((s.n_pages, pt // 16, 1), generator=gen, device=DEV).expand(-1, -1, 16).reshape(s.n_pages, pt) * _strength(d)
        at = (1, s.n_pages, pt, 1, 1) if c["tokens_first"] else (1, s.n_pages, 1, pt, 1)
        k.addcmul_(level.to(kind).view(at), u.to(kind))
    return k, v


def _rows(case, pool):
    """[layers][pages][kv_heads][page][dim] view of a pool."""
    return pool.transpose(2, 3) if case["tokens_first"] else pool


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _State()
    s.case = c = case
    lens, s.room = _ints(c["lens"]), _capacity(c)
    B, N, hq, h, d, pt, kind = len(lens), c["layers"], c["q_heads"], c["kv_heads"], c["dim"], c["page"], DTYPE[c["dtype"]]
    s.lens, s.batch = lens, B
    held = [-(-n // pt) for n in s.room]
    s.n_pages, s.pitch, s.slots = sum(held) + 1, max(1, max(held)), max(1, max(s.room))
    # the pages of a sequence lie anywhere in the pool
    order = torch.randperm(s.n_pages, generator=gen, device=DEV).to(torch.int32)
    s.table = torch.zeros((B, s.pitch), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(held):
        s.table[b, :n] = order[at:at + n]
        at += n
    u = torch.randn(d, generator=gen, device=DEV)
    u = u / u.norm()
    s.k, s.v = _pages(s, gen, u if c["mode"] == "attend" else None)
    length = torch.tensor(lens, dtype=torch.int32, device=DEV)[:, None].expand(B, h).contiguous()
    if c["uneven"]:   # whole chunks kept: a head more or fewer tokens than the next
        length = length - (torch.rand((B, h), generator=gen, device=DEV) * 40).int().clamp(max=length)
    s.length = length
    s.pos = s.weight = None
    if c["mode"] == "append":
        new = (_ints(c["new"]) * B)[:B] if len(_ints(c["new"])) == 1 else _ints(c["new"])
        s.new, T = new, sum(new)
        qkv = torch.randn((T, hq + 2 * h, d), generator=gen, device=DEV).to(kind)   # a fused projection's rows
        s.q, s.kn, s.vn = qkv[:, :hq], qkv[:, hq:hq + h], qkv[:, hq + h:]
        s.seq = torch.repeat_interleave(torch.arange(B, device=DEV), torch.tensor(new, device=DEV))
        s.nth = torch.cat([torch.arange(n, device=DEV) for n in new])
        # far into a long prompt: compression has left fewer slots than positions
        first = torch.randint(0, 200000, (B,), generator=gen, device=DEV)
        s.positions = (first[s.seq] + s.nth).to(torch.int32)
        s.q_norm, s.k_norm = ((1 + 0.2 * torch.randn(d, generator=gen, device=DEV)).to(kind) if c["norm"] else None for _ in range(2))
        s.eps = 1e-6
        r = c["rotary"]
        s.freq = (500000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)).float() if r else None
        s.q_out = torch.zeros((T, hq, d), dtype=kind, device=DEV)
        s.length_out = torch.zeros_like(length)
        s.pos = torch.zeros((B, h, s.slots), dtype=torch.int32, device=DEV)
        s.weight = torch.ones((B, h, s.slots), device=DEV) if c["weights"] else None
    elif c["mode"] == "attend":
        s.q = (torch.randn((B, hq, d), generator=gen, device=DEV) + u * _strength(d)).to(kind)
        s.out = torch.zeros((B, hq, d), device=DEV)
        s.lse = torch.zeros((B, hq), device=DEV)
        s.weight = torch.rand((B, h, s.slots), generator=gen, device=DEV) if c["weights"] else None
    elif c["mode"] == "compact":
        _prepare_compact(s, gen)
    else:
        # what accumulated weights look like: most tokens little, some much; slots of earlier evictions in any order
        n = N * B * h * s.slots
        s.start = torch.empty(2 * n + N * B * h, dtype=torch.int32, device=DEV)
        s.live = torch.empty_like(s.start)
        s.pos, s.weight = s.live[:n].view(N, B, h, s.slots), s.live[n:2 * n].view(torch.float32).view(N, B, h, s.slots)
        s.length_live = s.live[2 * n:].view(N, B, h)
        old = torch.rand((N, B, h, s.slots), generator=gen, device=DEV).argsort(-1)
        new = torch.arange(s.slots, device=DEV)
        fresh = new >= torch.minimum(length, torch.tensor(c["budget"], device=DEV, dtype=torch.int32))[None, ..., None]
        s.start[:n] = (torch.where(fresh, new + 4 * s.slots, 3 * old)).to(torch.int32).reshape(-1)
        s.start[n:2 * n].view(torch.float32).copy_(torch.randn(n, generator=gen, device=DEV).mul_(2).exp_())
        s.start[2 * n:] = length.expand(N, B, h).reshape(-1)
        s.budget = [c["budget"]] * B
    if own:
        import paper_2502_00299_amd as ckv
        p = c["page"] * h * d
        stride = (p, d, h * d) if c["tokens_first"] else (p, pt * d, d)
        s.ckv, s.kinds = ckv, {"bf16": ckv.BF16, "f16": ckv.F16, "f32": ckv.F32}
        s.handle = ckv.Pages(hq, h, d, s.kinds[c["dtype"]], pt, s.n_pages, s.room, *stride, table_pitch=s.pitch, slot_pitch=s.slots)
        s.ks, s.vs = list(s.k.unbind(0)), list(s.v.unbind(0))
        need = 0
        if c["mode"] == "attend":
            need = ckv.chunkkv_paged_decode_workspace_bytes(s.handle, c["weights"])
        elif c["mode"] == "evict":
            need = ckv.chunkkv_paged_evict_workspace_bytes(s.handle, N, s.budget)
        s.ws = torch.empty(max(256, need), dtype=torch.uint8, device=DEV)
        if c["mode"] == "compact":
            s.prob = ckv.Problem(hq, h, d, c["window"], c["chunk"], s.kinds[c["dtype"]], lens, s.keep, [sum(lens[:b]) * h * d for b in range(B)], d, h * d,
                                 sel_cap=s.sel_cap, score_cap=s.score_cap)
    return s


def _prepare_compact(s, gen):
    """Full caches packed [tokens][kv_heads][dim], and a selection of chunks as the library's calls write it."""
    c, lens, B = s.case, s.lens, s.batch
    h, d, w, size, N, kind = c["kv_heads"], c["dim"], c["window"], c["chunk"], c["layers"], DTYPE[c["dtype"]]
    G = -(-N // c["reuse"])
    s.keep = [m - w for m in s.room]
    s.sel_cap = max(-(-n // size) for n in s.keep) + 1
    s.score_cap = max(-(-(n - w) // size) for n in lens)
    s.full_k, s.full_v = ([torch.empty((sum(lens), h, d), dtype=kind, device=DEV).normal_(generator=gen) for _ in range(N)] for _ in range(2))
    s.sel_chunk = torch.zeros((G, B, h, s.sel_cap), dtype=torch.int32, device=DEV)
    s.sel_len = torch.zeros_like(s.sel_chunk)
    s.sel_count = torch.zeros((G, B, h), dtype=torch.int32, device=DEV)
    for b, n in enumerate(lens):
        m = -(-s.keep[b] // size)
        if m == 0:
            continue
        whole = (n - w) // size   # the ragged last chunk stays out: every chunk but the cut one is whole
        pick = torch.rand((G, h, whole), generator=gen, device=DEV).argsort(-1)[..., :m].sort(-1).values
        s.sel_chunk[:, b, :, :m] = pick.to(torch.int32)
        s.sel_len[:, b, :, :m] = size
        s.sel_len[:, b, :, m // 2] = s.keep[b] - (m - 1) * size
        s.sel_count[:, b] = m
    s.importance = [torch.rand((B, h, s.score_cap * size), generator=gen, device=DEV) for _ in range(G)] if c["weights"] else None
    s.length_out = torch.zeros((N, B, h), dtype=torch.int32, device=DEV)
    s.pos = torch.zeros((N, B, h, s.slots), dtype=torch.int32, device=DEV)
    s.weight = torch.zeros((N, B, h, s.slots), device=DEV) if c["weights"] else None


# ---- one pass -----------------------------------------------------------------------------------------------------


def _bits(x):
    """Rows that are copied are compared as the bits they are."""
    return x.view(torch.int16) if x.element_size() == 2 else x.view(torch.int32)


def run(s):
    return {"append": _append, "attend": _attend, "compact": _compact, "evict": _evict}[s.case["mode"]](s)


def _append(s):
    c = s.case
    if own:
        s.ckv.chunkkv_paged_append(s.handle, s.new, s.q, s.kn, s.vn, s.positions, s.q_norm, s.k_norm, s.eps, s.freq, c["interleaved"], s.q_out, s.table,
                                   s.ks[0], s.vs[0], s.length, s.length_out, s.pos, s.weight)
    else:
        pt, kind = c["page"], DTYPE[c["dtype"]]

        def turned(x, norm):
            x = x.float()
            if norm is not None:
                x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + s.eps) * norm.float()
            if s.freq is None:
                return x.to(kind)
            angle = (s.positions.double()[:, None] * s.freq.double())[:, None]
            cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
            r = c["rotary"]
            a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
            y, z = a * cos - b * sin, b * cos + a * sin
            both = torch.stack((y, z), -1).flatten(-2) if c["interleaved"] else torch.cat((y, z), -1)
            return torch.cat((both, x[..., r:]), -1).to(kind)

        s.q_out.copy_(turned(s.q, s.q_norm))
        heads = torch.arange(c["kv_heads"], device=DEV)
        slot = s.length.long()[s.seq] + s.nth[:, None]                 # [tokens][kv_heads]
        page = s.table.long()[s.seq[:, None], slot // pt]
        _rows(c, s.k)[0].index_put_((page, heads, slot % pt), turned(s.kn, s.k_norm))
        _rows(c, s.v)[0].index_put_((page, heads, slot % pt), s.vn)
        s.pos.index_put_((s.seq[:, None], heads, slot), s.positions[:, None].expand_as(slot))
        if s.weight is not None:
            s.weight.index_put_((s.seq[:, None], heads, slot), torch.zeros((), device=DEV))
        s.length_out.copy_(s.length + torch.bincount(s.seq, minlength=s.batch).int()[:, None])
    return {"q": s.q_out, "k": s.k, "v": _bits(s.v), "length": s.length_out, "pos": s.pos, "weight": s.weight}


def _gathered(s, pool, dtype):
    """[batch][kv_heads][slots][dim] of one layer, slots a whole number of pages."""
    x = _rows(s.case, pool)[0][s.table.long()]                        # [batch][pages][kv_heads][page][dim]
    return x.transpose(1, 2).flatten(2, 3).to(dtype)


def _attend(s):
    c = s.case
    if own:
        s.ckv.chunkkv_paged_decode_attention(s.handle, s.table, s.length, s.q, s.ks[0], s.vs[0], s.out, s.lse, s.weight, s.ws)
    else:
        h, d = c["kv_heads"], c["dim"]
        k, v = _gathered(s, s.k, torch.float32), _gathered(s, s.v, torch.float32)
        q = s.q.float().view(s.batch, h, -1, d)
        here = (torch.arange(k.shape[2], device=DEV) < s.length[..., None])[:, :, None]
        x = (torch.matmul(q, k.transpose(2, 3)) * d ** -0.5).masked_fill(~here, float("-inf"))
        top = x.amax(-1, keepdim=True).clamp(min=-3e38)
        p = torch.exp(x - top)
        total = p.sum(-1, keepdim=True)
        p = p / total.clamp(min=1e-30)
        s.out.copy_(torch.matmul(p, v).flatten(1, 2))
        s.lse.copy_((top + torch.log(total)).flatten(1))
        if s.weight is not None:
            s.weight += p.sum(2)[..., :s.slots]
    return {"out": s.out, "lse": s.lse, "weight": s.weight}


def _compact(s):
    c = s.case
    if own:
        s.ckv.chunkkv_paged_compact(s.prob, s.handle, c["reuse"], s.full_k, s.full_v, s.sel_chunk, s.sel_len, s.sel_count, s.importance, s.table, s.ks, s.vs,
                                    s.length_out, s.pos, s.weight)
    else:
        h, d, w, size, N, pt = c["kv_heads"], c["dim"], c["window"], c["chunk"], c["layers"], c["page"]
        i = torch.arange(size, device=DEV)
        live = (torch.arange(s.sel_cap, device=DEV) < s.sel_count[..., None])[..., None] & (i < s.sel_len[..., None])
        token = (s.sel_chunk[..., None].long() * size + i).flatten(-2)
        ends = torch.tensor(s.lens, device=DEV)
        window = (ends[:, None] - w + torch.arange(w, device=DEV))[None, :, None].expand(*token.shape[:3], w)
        token, live = torch.cat((token, window), -1), torch.cat((live.flatten(-2), torch.ones_like(window, dtype=torch.bool)), -1)
        group, b, head, e = live.nonzero(as_tuple=True)                # in the order of the slots
        slot = (live.cumsum(-1) - 1)[group, b, head, e]
        token = token[group, b, head, e]
        page = s.table.long()[b, slot // pt]
        row = (torch.cumsum(ends, 0) - ends)[b] + token
        in_group = torch.arange(N, device=DEV)[:, None] // c["reuse"] == group
        layer, at = in_group.nonzero(as_tuple=True)
        place = (layer, page[at], head[at], slot[at] % pt)
        _rows(c, s.k).index_put_(place, torch.stack(s.full_k)[layer, row[at], head[at]])
        _rows(c, s.v).index_put_(place, torch.stack(s.full_v)[layer, row[at], head[at]])
        s.pos[layer, b[at], head[at], slot[at]] = token[at].int()
        if s.weight is not None:
            past = torch.cat((torch.stack(s.importance), torch.zeros((len(s.importance), s.batch, h, w), device=DEV)), -1)
            inside = token < ends[b] - w
            s.weight[layer, b[at], head[at], slot[at]] = torch.where(inside, past[group, b, head, torch.where(inside, token, past.shape[-1] - 1)], 0.0)[at]
        s.length_out.copy_(live.sum(-1).int()[torch.arange(N, device=DEV) // c["reuse"]])
    return {"k": _bits(s.k), "v": _bits(s.v), "length": s.length_out, "pos": s.pos, "weight": s.weight}


def _evict(s):
    c = s.case
    s.live.copy_(s.start)   # as it is before the eviction, so that the next pass has the same to do
    if own:
        s.ckv.chunkkv_paged_evict(s.handle, s.budget, c["recent"], s.table, s.ks, s.vs, s.length_live, s.pos, s.weight, s.ws)
    else:
        slot = torch.arange(s.slots, device=DEV)
        held = slot < s.length_live[..., None]
        newest = torch.where(held, s.pos, -1).amax(-1, keepdim=True)
        key = torch.where(s.pos > newest - c["recent"], float("inf"), s.weight).masked_fill(~held, float("-inf"))
        left = s.length_live.clamp(max=c["budget"])
        ranked = torch.sort(key, dim=-1, descending=True, stable=True).indices
        stays = torch.zeros_like(held).scatter_(-1, ranked, slot < left[..., None])
        inside = slot < left[..., None]
        n, b, h, to = (inside & ~stays).nonzero(as_tuple=True)
        source = (stays & ~inside).nonzero(as_tuple=True)[3]          # as many, head for head
        table, pt = s.table.long(), c["page"]
        k, v = _rows(c, s.k), _rows(c, s.v)
        place, taken = (n, table[b, to // pt], h, to % pt), (n, table[b, source // pt], h, source % pt)
        k.index_put_(place, k[taken])
        v.index_put_(place, v[taken])
        s.pos[n, b, h, to] = s.pos[n, b, h, source]
        s.weight[n, b, h, to] = s.weight[n, b, h, source]
        s.length_live.copy_(left)
    return {"k": _bits(s.k), "v": _bits(s.v), "length": s.length_live, "pos": s.pos, "weight": s.weight}


# ---- what the definition gives in 64 bits ---------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    c, pt = case, case["page"]
    if c["mode"] == "append":
        return _exact_append(s)
    if c["mode"] == "attend":
        g = c["q_heads"] // c["kv_heads"]
        out, lse = torch.zeros_like(s.out, dtype=torch.float64), torch.full_like(s.lse, float("-inf"), dtype=torch.float64)
        weight = None if s.weight is None else s.weight.double()
        k, v = _rows(c, s.k)[0], _rows(c, s.v)[0]
        for b in range(s.batch):
            pages = s.table[b, :max(1, -(-s.room[b] // pt))].long()
            for h in range(c["kv_heads"]):
                n = int(s.length[b, h])
                if n == 0:
                    continue
                kk, vv = (x[pages, h].reshape(-1, c["dim"])[:n].double() for x in (k, v))
                heads = slice(h * g, (h + 1) * g)
                x = s.q[b, heads].double() @ kk.t().contiguous() / math.sqrt(c["dim"])
                lse[b, heads] = torch.logsumexp(x, 1)
                p = torch.exp(x - lse[b, heads, None])
                out[b, heads] = p @ vv
                if weight is not None:
                    weight[b, h, :n] += p.sum(0)
        return {"out": out, "lse": lse, "weight": weight}
    if c["mode"] == "compact":
        if s.weight is None:
            return None
        # the importance of the tokens that a head keeps, in ascending order, then the window, which has none
        want = torch.zeros(s.weight.shape, dtype=torch.float64)
        count, chunk, length = s.sel_count.cpu(), s.sel_chunk.cpu(), s.sel_len.cpu()
        past = [x.cpu().double() for x in s.importance]
        for g in range(len(past)):
            for b in range(s.batch):
                for h in range(c["kv_heads"]):
                    tokens = [int(chunk[g, b, h, e]) * c["chunk"] + i for e in range(int(count[g, b, h])) for i in range(int(length[g, b, h, e]))]
                    want[g * c["reuse"]:(g + 1) * c["reuse"], b, h, :len(tokens)] = past[g][b, h, tokens]
        return {"weight": want}
    # eviction copies: weights that stay are the ones that were
    before, held = s.start, s.length.cpu()
    n = (before.numel() - s.length_live.numel()) // 2
    shape = s.weight.shape
    if n > 3_000_000:
        return None
    pos, want = before[:n].view(shape).cpu().numpy(), before[n:2 * n].view(torch.float32).view(shape).cpu().double().numpy()
    for i in range(c["layers"]):
        for b in range(s.batch):
            for h in range(c["kv_heads"]):
                m = int(held[b, h])
                if m <= c["budget"]:
                    continue
                p, w = pos[i, b, h, :m].tolist(), want[i, b, h, :m].tolist()
                since = max(p) - c["recent"]
                best = sorted(range(m), key=lambda j: (-math.inf if p[j] > since else -w[j], j))[:c["budget"]]
                stay = set(best)
                free = [j for j in range(c["budget"]) if j not in stay]
                for to, j in zip(free, sorted(j for j in best if j >= c["budget"])):
                    want[i, b, h, to] = w[j]
    return {"weight": torch.from_numpy(want)}


def _exact_append(s):
    c, pt, r = s.case, s.case["page"], s.case["rotary"]

    def turned(x, norm):
        y = x.double()
        if norm is not None:
            y = y / torch.sqrt((y * y).sum(-1, keepdim=True) / c["dim"] + s.eps) * norm.double()
        if r:
            i = torch.arange(r // 2, device=DEV)
            first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + r // 2)
            unit = torch.polar(torch.ones((), dtype=torch.float64, device=DEV).expand(len(x), r // 2), s.positions.double()[:, None] * s.freq.double()[None])
            z = torch.complex(y[..., first], y[..., second]) * unit[:, None]
            y = y.clone()
            y[..., first], y[..., second] = z.real, z.imag
        return y

    pool = s.k.double()
    k, rows = turned(s.kn, s.k_norm), _rows(c, pool)[0]
    at = 0
    for b, n in enumerate(s.new):
        for h in range(c["kv_heads"]):
            slot = int(s.length[b, h]) + torch.arange(n, device=DEV)
            rows[s.table[b].long()[slot // pt], h, slot % pt] = k[at:at + n, h]
        at += n
    return {"q": turned(s.q, s.q_norm), "k": pool, "weight": None}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    lens, room = _ints(case["lens"]), _capacity(case)
    hq, h, d, N = case["q_heads"], case["kv_heads"], case["dim"], case["layers"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["mode"] == "append":
        T = sum(room) - sum(lens)
        moved = T * (2 * (hq + 2 * h) * d * e + 4 + h * (8 if case["weights"] else 4))
        return {"bytes": float(moved), "flops": float(T * (hq + h) * d * 8)}
    if case["mode"] == "attend":
        n = sum(lens) - (20 * len(lens) if case["uneven"] else 0)
        n = max(n, len(lens))
        moved = h * n * (2 * d * e + (8 if case["weights"] else 0)) + len(lens) * hq * (d * e + 4 * d + 4)
        return {"bytes": float(moved), "flops": float(4 * hq * n * d)}
    if case["mode"] == "compact":
        entries = sum(-(-(m - case["window"]) // case["chunk"]) for m in room)
        moved = N * h * sum(room) * (4 * d * e + 4) + 8 * h * entries * -(-N // case["reuse"]) + (8 * N * h * sum(room) if case["weights"] else 0)
        return {"bytes": float(moved), "flops": 0.0}
    m, moved = case["budget"], 0.0
    for n in lens:
        out, new = max(0, n - m), min(case["recent"], max(0, n - m))
        # of the slots past the budget: the protected ones, and of the others as many as stay everywhere
        movers = new + (out - new) * max(0, m - case["recent"]) / max(1, n - case["recent"]) if out else 0
        moved += N * h * (8 * n * (out > 0) + movers * (4 * d * e + 8))
    return {"bytes": float(max(moved, 4 * N * h * len(lens))), "flops": 0.0}
