"""Operators around a cache that many queries read, as cases that can be timed and compared.

A document's cache is made once and read by many: its keys and window queries are rotated by position (`rotate`), the tokens of a
question attend to the whole of it, or a decoder's to an encoder's states (`cross`: no order between queries and states, lengths that
have nothing to do with each other, padding that a mask takes out), and a batch of sequences goes on behind it token by token, each
with pages of its own (`shared`: the document's pages are read once for all sequences that share them).

Keys and queries have the structure of the repository's generator: N(0,1) and a shared direction whose strength is graded over runs
of tokens (about 2 nats of the logit), so attention is uneven as over a prompt.
"""
import math

import torch

own = False

DEV = "cuda:0"
DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


def _case(name, mode, **kw):
    case = dict(name=name, mode=mode, q_heads=32, kv_heads=8, dim=128, dtype="bf16", lse=False,
                seqs=1, tokens=1, rotary=128, interleaved=False, magnitude=1.0, to_cache=False,
                queries="1", states="1", layout="heads", holes=0.0,
                prefix="1", sharing="1", lens="1", page=16, tokens_first=False, uneven=False)
    case.update(kw)
    return case


def listed():
    return [
        # a decoding step of eight sequences: every token's queries and keys, rows of a fused projection
        _case("rotate_step_b8", "rotate", tokens=8),
        # three prompts of odd length, fp16, half of the head in neighbouring pairs, positions far into a scaled context
        _case("rotate_part_f16", "rotate", seqs=3, tokens=1501, q_heads=28, kv_heads=4, dtype="f16", rotary=64, interleaved=True, magnitude=1.1386),
        # a 32K prompt, frequencies and magnitude scaled; keys go from the projection's order to that of a cache
        _case("rotate_prompt_32k", "rotate", tokens=32768, magnitude=1.2079, to_cache=True),
        # one decoder token of eight sequences over their padded encoder states
        _case("cross_token_b8", "cross", queries="1 1 1 1 1 1 1 1", states="1500 1311 740 1500 96 1203 1499 0", q_heads=16, kv_heads=16, dim=64, layout="padded"),
        # the tokens of one question over a 128K prompt kept at 10 %
        _case("cross_question", "cross", queries="61", states="13171", lse=True),
        # fp32, ragged, packed; a sequence without queries, one without states, one of one token and one state
        _case("cross_ragged_f32", "cross", queries="300 1 77 0 1 513", states="2049 777 0 500 1 1031", q_heads=16, kv_heads=4, dim=64, dtype="f32", layout="packed", lse=True),
        # a batch of an encoder-decoder, fp16, padded, with holes in the mask
        _case("cross_batch_f16", "cross", queries="512 512 512 512 512 512 512 512", states="2048 1999 1024 2048 333 1777 2000 2048", q_heads=16, kv_heads=16, dim=64,
              dtype="f16", layout="padded", holes=0.1),
        # a prompt's chunk over a cache of 16K states: as many products as a prefill
        _case("cross_chunk_16k", "cross", queries="4096", states="16384"),
        # eight answers to an 8K prompt kept at 10 %, their first tokens
        _case("shared_b8_kept", "shared", prefix="848", sharing="8", lens="1 7 12 33 2 64 5 20"),
        # fp32 caches, two prefixes, heads of unequal length
        _case("shared_f32_d64", "shared", prefix="3111 1024", sharing="4 3", lens="75 1 300 0 17 640 16", q_heads=16, kv_heads=4, dim=64, dtype="f32", page=48,
              uneven=True, lse=True),
        # three documents with their readers, fp16, one of them read by one alone, tokens of all heads together in a page
        _case("shared_groups_f16", "shared", prefix="20995 4096 10460", sharing="5 1 17", lens=" ".join(str(40 + (i * 397) % 701) for i in range(23)), q_heads=28,
              kv_heads=4, dtype="f16", page=32, tokens_first=True),
        # 64 sequences behind a 128K document with its full cache
        _case("shared_b64_128k", "shared", prefix="131072", sharing="64", lens=" ".join(str(100 + (i * 4733) % 901) for i in range(64)), page=128),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _text(numbers):
    return " ".join(map(str, numbers))


def draw(rng):
    mode = rng.choice(["rotate", "cross", "cross", "shared", "shared"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    q_heads, kv_heads = rng.choice([(32, 8), (32, 8), (28, 4), (16, 4), (8, 8), (16, 16), (4, 2), (64, 8)])
    dim = rng.choice([128, 128, 64])
    case = _case("", mode, q_heads=q_heads, kv_heads=kv_heads, dim=dim, dtype=dtype, lse=rng.random() < 0.4)
    del case["name"]
    slow = 16 if dtype == "f32" else 1                   # fp32 products have a sixteenth of the rate
    if mode == "rotate":
        seqs = rng.choice([1, 1, 2, 3, 8])
        tokens = _log_uniform(rng, 1, 32768 / seqs)
        while seqs * tokens * (q_heads + kv_heads) * dim > (1.6e8 if dtype != "f32" else 8e7):
            tokens //= 2
        case.update(seqs=seqs, tokens=tokens, rotary=rng.choice([dim, dim, dim // 2, 16]), interleaved=rng.random() < 0.4,
                    magnitude=rng.choice([1.0, round(rng.uniform(1.0, 1.5), 4)]), to_cache=rng.random() < 0.5)
        return case
    if mode == "cross":
        batch = rng.choice([1, 1, 2, 5, 8])
        queries = [1] * batch if rng.random() < 0.3 else [max(1, int(_log_uniform(rng, 1, 4096) * rng.uniform(0.1, 1.0))) for _ in range(batch)]
        top = _log_uniform(rng, 1, 131072)
        states = [top] + [int(top * rng.uniform(0.0, 1.0)) for _ in range(batch - 1)]
        while (4.0 * q_heads * dim * sum(a * b for a, b in zip(queries, states)) > 1.0e12 / slow or batch * max(states) * kv_heads * dim > 1.3e8 / (1 + slow // 16)):
            if max(queries) > 1 and rng.random() < 0.5:
                queries = [max(1, n // 2) for n in queries]
            else:
                states = [n // 2 for n in states]
        if max(states) == 0:
            states[0] = 1
        layout = rng.choice(["heads", "packed", "padded"])
        case.update(queries=_text(queries), states=_text(states), layout=layout, holes=rng.choice([0.0, 0.1, 0.5]) if layout == "padded" else 0.0)
        return case
    groups = rng.choice([1, 1, 1, 2, 4])
    sharing = [_log_uniform(rng, 1, 64 / groups) for _ in range(groups)]
    top = _log_uniform(rng, 16, 131072)
    prefix = [top] + [int(top * rng.uniform(0.02, 1.0)) for _ in range(groups - 1)]
    most = _log_uniform(rng, 1, 2000)
    lens = [rng.randint(0, most) for _ in range(sum(sharing))]
    row = kv_heads * dim * (1 + slow // 16)
    while sum(prefix) * row > 1.3e8:
        prefix = [max(1, n // 2) for n in prefix]
    while sum(lens) * row > 4e7:
        lens = [n // 2 for n in lens]
    while 4.0 * q_heads * dim * sum(a * b for a, b in zip(prefix, sharing)) > 4.0e11 / slow:
        prefix = [max(1, n // 2) for n in prefix]
    case.update(prefix=_text(prefix), sharing=_text(sharing), lens=_text(lens), page=rng.choice([16, 16, 32, 48, 64, 128, 256]),
                tokens_first=rng.random() < 0.3, uneven=rng.random() < 0.3)
    return case


def _ints(text):
    return [int(x) for x in text.split()]


# ---- inputs -------------------------------------------------------------------------------------------------------


class _State:
    pass


def _strength(d):
    return math.sqrt(2.0 * math.sqrt(d))


def _keys(shape, axis, gen, u, kind):
    """N(0,1) keys with runs of 16 along `axis` that share the direction u to a graded degree."""
    k = torch.empty(shape, dtype=kind, device=DEV).normal_(generator=gen)
    n = shape[axis]
    level = torch.randn(-(-n // 16) + 1, generator=gen, device=DEV).repeat_interleave(16)[:n] * _strength(shape[-1])
    return k.addcmul_(level.to(kind).view([-1 if i == axis else 1 for i in range(len(shape))]), u.to(kind))


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s = _State()
    s.case = case
    s.kind = DTYPE[case["dtype"]]
    s.ckv = None
    if own:
        import paper_2502_00299_amd as ckv
        s.ckv, s.code = ckv, {"bf16": ckv.BF16, "f16": ckv.F16, "f32": ckv.F32}[case["dtype"]]
    {"rotate": _prepare_rotate, "cross": _prepare_cross, "shared": _prepare_shared}[case["mode"]](s, gen)
    return s


def _prepare_rotate(s, gen):
    c = s.case
    n, t, hq, h, d, r = c["seqs"], c["tokens"], c["q_heads"], c["kv_heads"], c["dim"], c["rotary"]
    qkv = torch.randn((n, t, hq + 2 * h, d), generator=gen, device=DEV).to(s.kind)   # a fused projection's rows
    s.q, s.k = qkv[:, :, :hq], qkv[:, :, hq:hq + h]
    first = torch.randint(0, 200000, (n, 1), generator=gen, device=DEV)
    s.positions = (first + torch.arange(t, device=DEV)).to(torch.int32)
    # frequencies of a context four times as long as the trained one: those that turn often enough stay, the slowest are divided
    freq = 500000.0 ** (-torch.arange(0, r, 2, device=DEV, dtype=torch.float64) / r)
    if c["magnitude"] != 1.0:
        stay = ((8192.0 * freq / (2 * math.pi) - 1.0) / 31.0).clamp(0.0, 1.0)
        freq = freq * stay + freq / 4.0 * (1.0 - stay)
    s.freq = freq.float()
    s.q_out = torch.zeros((n, t, hq, d), dtype=s.kind, device=DEV)
    s.k_out = torch.zeros((n, h, t, d), dtype=s.kind, device=DEV).transpose(1, 2) if c["to_cache"] else torch.zeros((n, t, h, d), dtype=s.kind, device=DEV)


def _prepare_cross(s, gen):
    c = s.case
    hq, h, d, kind = c["q_heads"], c["kv_heads"], c["dim"], s.kind
    s.queries, s.states = _ints(c["queries"]), _ints(c["states"])
    B, T, most = len(s.queries), sum(s.queries), max(s.states)
    u = torch.randn(d, generator=gen, device=DEV)
    u = u / u.norm()
    s.q = (torch.randn((T, hq, d), generator=gen, device=DEV) + u * _strength(d)).to(kind)
    s.first = [sum(s.queries[:b]) for b in range(B)]
    s.mask = None
    if c["layout"] == "padded":      # [B][longest][heads][d], what is behind a sequence's states masked out, and holes
        shape, axis = (B, most, h, d), 1
        s.mask = torch.arange(most, device=DEV) < torch.tensor(s.states, device=DEV)[:, None]
        s.mask &= torch.rand((B, most), generator=gen, device=DEV) >= c["holes"]
        s.rooms, s.base, s.strides = [most] * B, [b * most * h * d for b in range(B)], (d, h * d)
    elif c["layout"] == "packed":    # [all states][heads][d]
        shape, axis = (sum(s.states), h, d), 0
        s.rooms, s.base, s.strides = s.states, [sum(s.states[:b]) * h * d for b in range(B)], (d, h * d)
    else:                            # [B][heads][longest][d]
        shape, axis = (B, h, most, d), 2
        s.rooms, s.base, s.strides = s.states, [b * h * most * d for b in range(B)], (most * d, d)
    s.k = _keys(shape, axis, gen, u, kind)
    s.v = torch.empty(shape, dtype=kind, device=DEV).normal_(generator=gen)
    s.out = torch.zeros((T, hq, d), dtype=kind, device=DEV)
    s.lse = torch.zeros((T, hq), device=DEV) if c["lse"] else None
    if s.ckv:
        s.plan = s.ckv.Cross(hq, h, d, s.code, s.queries, s.rooms, s.base, *s.strides)
        s.ws = torch.empty(max(256, s.ckv.chunkkv_cross_workspace_bytes(s.plan)), dtype=torch.uint8, device=DEV)


def _prepare_shared(s, gen):
    c = s.case
    hq, h, d, pt, kind = c["q_heads"], c["kv_heads"], c["dim"], c["page"], s.kind
    s.prefix, s.sharing, s.lens = _ints(c["prefix"]), _ints(c["sharing"]), _ints(c["lens"])
    B = len(s.lens)
    rooms = s.prefix + s.lens
    held = [-(-n // pt) for n in rooms]
    n_pages, pitch = sum(held) + 1, max(1, max(held))
    # the pages of a prefix or a sequence lie anywhere in the pool
    order = torch.randperm(n_pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.zeros((len(rooms), pitch), dtype=torch.int32, device=DEV)
    at = 0
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    s.prefix_table, s.table = table[:len(s.prefix)].contiguous(), table[len(s.prefix):].contiguous()
    u = torch.randn(d, generator=gen, device=DEV)
    u = u / u.norm()
    length = torch.tensor(rooms, dtype=torch.int32, device=DEV)[:, None].expand(len(rooms), h).contiguous()
    if c["uneven"]:   # whole chunks kept: a head more or fewer tokens than the next
        length = length - (torch.rand(length.shape, generator=gen, device=DEV) * 40).int().clamp(max=length)
    s.prefix_len, s.length = length[:len(s.prefix)].contiguous(), length[len(s.prefix):].contiguous()
    shape = (n_pages, pt, h, d) if c["tokens_first"] else (n_pages, h, pt, d)
    s.k = torch.empty(shape, dtype=kind, device=DEV).normal_(generator=gen)
    s.v = torch.empty(shape, dtype=kind, device=DEV).normal_(generator=gen)
    level = torch.randn((n_pages, pt // 16, 1), generator=gen, device=DEV).expand(-1, -1, 16).reshape(n_pages, pt) * _strength(d)
    s.k.addcmul_(level.to(kind).view((n_pages, pt, 1, 1) if c["tokens_first"] else (n_pages, 1, pt, 1)), u.to(kind))
    s.q = (torch.randn((B, hq, d), generator=gen, device=DEV) + u * _strength(d)).to(kind)
    s.out = torch.zeros((B, hq, d), dtype=kind, device=DEV)
    s.lse = torch.zeros((B, hq), device=DEV) if c["lse"] else None
    if s.ckv:
        p = pt * h * d
        stride = (p, d, h * d) if c["tokens_first"] else (p, pt * d, d)
        s.whole, s.pages = (s.ckv.Pages(hq, h, d, s.code, pt, n_pages, room, *stride, table_pitch=pitch) for room in (s.prefix, s.lens))
        s.ws = torch.empty(max(256, s.ckv.chunkkv_shared_decode_workspace_bytes(s.whole, s.pages, s.sharing)), dtype=torch.uint8, device=DEV)


# ---- one pass -----------------------------------------------------------------------------------------------------


def run(s):
    return {"rotate": _rotate, "cross": _cross, "shared": _shared}[s.case["mode"]](s)


def _rotate(s):
    c = s.case
    if own:
        s.ckv.chunkkv_rotate(s.q, s.k, s.positions, s.freq, c["interleaved"], c["magnitude"], s.q_out, s.k_out)
    else:
        r = c["rotary"]
        angle = (s.positions.double()[..., None] * s.freq.double())[:, :, None]
        cos, sin = (torch.cos(angle) * c["magnitude"]).float(), (torch.sin(angle) * c["magnitude"]).float()
        for x, to in ((s.q, s.q_out), (s.k, s.k_out)):
            x = x.float()
            a, b = (x[..., 0:r:2], x[..., 1:r:2]) if c["interleaved"] else (x[..., :r // 2], x[..., r // 2:r])
            y, z = a * cos - b * sin, b * cos + a * sin
            both = torch.stack((y, z), -1).flatten(-2) if c["interleaved"] else torch.cat((y, z), -1)
            to.copy_(torch.cat((both, x[..., r:]), -1))
    return {"q": s.q_out, "k": s.k_out}


def _states(s, x, b):
    """[kv_heads][states][dim] of sequence b."""
    c = s.case
    return x.view(-1).as_strided((c["kv_heads"], s.rooms[b], c["dim"]), (*s.strides, 1), s.base[b])


def _softmax_parts(x):
    """Maximum, exponentials relative to it and their sum; rows without an entry sum to 0."""
    top = x.amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(x - top)
    return top, p, p.sum(-1, keepdim=True)


def _cross(s):
    c = s.case
    if own:
        s.ckv.chunkkv_cross_attention(s.plan, None, s.mask, s.q, s.k, s.v, s.out, s.lse, s.ws)
    else:
        hq, h, d = c["q_heads"], c["kv_heads"], c["dim"]
        for b, (n, m) in enumerate(zip(s.queries, s.rooms)):
            if n == 0:
                continue
            if m == 0:
                s.out[s.first[b]:s.first[b] + n] = 0
                if s.lse is not None:
                    s.lse[s.first[b]:s.first[b] + n] = float("-inf")
                continue
            k, v = _states(s, s.k, b).float().transpose(1, 2), _states(s, s.v, b).float()
            step = max(1, (1 << 28) // (hq * m))
            for t in range(0, n, step):
                at = slice(s.first[b] + t, s.first[b] + min(n, t + step))
                q = s.q[at].float().unflatten(1, (h, -1)).permute(1, 0, 2, 3)            # [kv_heads][tokens][group][dim]
                x = torch.matmul(q.flatten(1, 2), k) * d ** -0.5
                if s.mask is not None:
                    x = x.masked_fill(~s.mask[b], float("-inf"))
                top, p, total = _softmax_parts(x)
                o = torch.matmul(p, v) / total.clamp(min=1e-30)
                s.out[at] = o.unflatten(1, q.shape[1:3]).permute(1, 0, 2, 3).flatten(1, 2).to(s.kind)
                if s.lse is not None:
                    s.lse[at] = (top + torch.log(total)).unflatten(1, q.shape[1:3])[..., 0].permute(1, 0, 2).flatten(1)
    return {"out": s.out, "lse": s.lse}


def _slots(s, pool, table):
    """[rows of the table][kv_heads][slots][dim] in fp32."""
    x = pool.transpose(1, 2) if s.case["tokens_first"] else pool
    return x[table.long()].transpose(1, 2).flatten(2, 3).float()


def _shared(s):
    c = s.case
    if own:
        s.ckv.chunkkv_shared_decode_attention(s.whole, s.pages, s.sharing, s.prefix_table, s.prefix_len, s.table, s.length, s.q, s.k, s.v, s.out, s.lse, s.ws)
    else:
        h, d, pt = c["kv_heads"], c["dim"], c["page"]
        at = 0
        for i, n in enumerate(s.sharing):
            rows, at = slice(at, at + n), at + n
            q = s.q[rows].float().unflatten(1, (h, -1))                                      # [sequences][kv_heads][group][dim]
            width, own_width = (max(1, -(-m // pt)) for m in (s.prefix[i], max(s.lens[rows])))
            k, v = (_slots(s, x, s.prefix_table[i:i + 1, :width])[0] for x in (s.k, s.v))
            ko, vo = (_slots(s, x, s.table[rows, :own_width]) for x in (s.k, s.v))
            x = torch.matmul(q.transpose(0, 1).flatten(1, 2), k.transpose(1, 2)) * d ** -0.5  # [kv_heads][sequences * group][slots]
            x = x.masked_fill(torch.arange(k.shape[1], device=DEV) >= s.prefix_len[i][:, None, None], float("-inf"))
            y = torch.matmul(q, ko.transpose(2, 3)) * d ** -0.5
            y = y.masked_fill(torch.arange(ko.shape[2], device=DEV) >= s.length[rows][:, :, None, None], float("-inf"))
            tops, parts, sums = zip(_softmax_parts(x), _softmax_parts(y))
            outs = (torch.matmul(parts[0], v), torch.matmul(parts[1], vo))
            tops, sums, outs = ((e[0].unflatten(1, (n, -1)).transpose(0, 1), e[1]) for e in (tops, sums, outs))
            top = torch.maximum(*tops)
            f = [torch.exp(t - top) for t in tops]
            total = sums[0] * f[0] + sums[1] * f[1]
            s.out[rows] = ((outs[0] * f[0] + outs[1] * f[1]) / total.clamp(min=1e-30)).flatten(1, 2).to(s.kind)
            if s.lse is not None:
                s.lse[rows] = (top + torch.log(total))[..., 0].flatten(1)
    return {"out": s.out, "lse": s.lse}


# ---- what the definition gives in 64 bits ---------------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "cross": _exact_cross, "shared": _exact_shared}[case["mode"]](s)


def _exact_rotate(s):
    c, r = s.case, s.case["rotary"]

    def turned(x):
        y = x.double().clone()
        i = torch.arange(r // 2, device=DEV)
        first, second = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + r // 2)
        angle = s.positions.double()[:, :, None, None] * s.freq.double()
        z = torch.complex(y[..., first], y[..., second]) * torch.polar(torch.full_like(angle, c["magnitude"]), angle)
        y[..., first], y[..., second] = z.real, z.imag
        return y

    return {"q": turned(s.q), "k": turned(s.k)}


def _attend(q, k, v, scale):
    """Outputs and log-sum-exps of rows q over keys k, in 64 bits."""
    if k.shape[0] == 0:
        return torch.zeros_like(q), torch.full(q.shape[:1], float("-inf"), dtype=torch.float64, device=DEV)
    x = q @ k.t() * scale
    z = torch.logsumexp(x, 1)
    return torch.exp(x - z[:, None]) @ v, z


def _exact_cross(s):
    c = s.case
    g, d = c["q_heads"] // c["kv_heads"], c["dim"]
    out, lse = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV), torch.zeros(s.out.shape[:2], dtype=torch.float64, device=DEV)
    for b, n in enumerate(s.queries):
        here = torch.arange(s.rooms[b], device=DEV) if s.mask is None else s.mask[b].nonzero()[:, 0]
        for i in range(c["kv_heads"]):
            k, v = (_states(s, x, b)[i][here].double() for x in (s.k, s.v))
            for t in range(0, n, 512):
                rows = slice(s.first[b] + t, s.first[b] + min(n, t + 512))
                o, z = _attend(s.q[rows, i * g:(i + 1) * g].double().flatten(0, 1), k, v, 1.0 / math.sqrt(d))
                out[rows, i * g:(i + 1) * g], lse[rows, i * g:(i + 1) * g] = o.view(-1, g, d), z.view(-1, g)
    return {"out": out, "lse": lse if s.lse is not None else None}


def _exact_shared(s):
    c, pt = s.case, s.case["page"]
    g, d = c["q_heads"] // c["kv_heads"], c["dim"]
    out, lse = torch.zeros(s.out.shape, dtype=torch.float64, device=DEV), torch.zeros(s.out.shape[:2], dtype=torch.float64, device=DEV)

    def rows(pool, table, i, n):
        x = pool[:, :, i] if c["tokens_first"] else pool[:, i]
        return x[table[:-(-n // pt)].long()].flatten(0, 1)[:n].double()

    at = 0
    for p, n in enumerate(s.sharing):
        for i in range(c["kv_heads"]):
            whole = [rows(x, s.prefix_table[p], i, int(s.prefix_len[p, i])) for x in (s.k, s.v)]
            for b in range(at, at + n):
                k, v = (torch.cat((w, rows(x, s.table[b], i, int(s.length[b, i])))) for w, x in zip(whole, (s.k, s.v)))
                out[b, i * g:(i + 1) * g], lse[b, i * g:(i + 1) * g] = _attend(s.q[b, i * g:(i + 1) * g].double(), k, v, 1.0 / math.sqrt(d))
        at += n
    return {"out": out, "lse": lse if s.lse is not None else None}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------


def work(case):
    hq, h, d = case["q_heads"], case["kv_heads"], case["dim"]
    e = 4 if case["dtype"] == "f32" else 2
    if case["mode"] == "rotate":
        T = case["seqs"] * case["tokens"]
        return {"bytes": float(T * (2 * (hq + h) * d * e + 4)), "flops": float(T * (hq + h) * case["rotary"] * 3)}
    if case["mode"] == "cross":
        queries, states = _ints(case["queries"]), _ints(case["states"])
        moved = sum(queries) * hq * (2 * d * e + (4 if case["lse"] else 0)) + 2 * h * d * e * sum(m for n, m in zip(queries, states) if n)
        moved += len(states) * max(states) if case["layout"] == "padded" else 0
        return {"bytes": float(moved), "flops": float(4 * hq * d * sum(n * m for n, m in zip(queries, states)))}
    prefix, sharing, lens = _ints(case["prefix"]), _ints(case["sharing"]), _ints(case["lens"])
    short = 20 if case["uneven"] else 0
    prefix, lens = [max(0, n - short) for n in prefix], [max(0, n - min(short, n // 2)) for n in lens]
    moved = len(lens) * hq * (2 * d * e + (4 if case["lse"] else 0)) + 2 * h * d * e * (sum(prefix) + sum(lens))
    return {"bytes": float(moved), "flops": float(4 * hq * d * (sum(n * m for n, m in zip(prefix, sharing)) + sum(lens)))}
