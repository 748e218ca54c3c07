"""Paged caches for the tests: pools full of NaN wherever no token is, tables whose unused entries point nowhere."""
import torch

import paper_2502_00299_amd as ckv

DEV = "cuda:0"
KIND = {ckv.F32: torch.float32, ckv.BF16: torch.bfloat16, ckv.F16: torch.float16}
HALF_STEP = {ckv.F32: 2.0 ** -24, ckv.BF16: 2.0 ** -8, ckv.F16: 2.0 ** -11}


class Cache:
    """Pools of `layers` layers on the host, [layers][pages][heads][page][dim]; device copies in either layout."""

    def __init__(self, gen, dtype, hq, hkv, d, page, room, lens, layers=1, tokens_first=False, spare=3, scale=0.0):
        self.dtype, self.hq, self.hkv, self.d, self.page, self.layers, self.tokens_first = dtype, hq, hkv, d, page, layers, tokens_first
        self.room, self.batch = list(room), len(room)
        held = [-(-n // page) for n in room]
        self.n_pages = sum(held) + spare
        pitch, slots = max([1] + held) + 1, max([1] + list(room)) + 3
        self.table = torch.full((self.batch, pitch), -(1 << 30), dtype=torch.int32)
        order = torch.randperm(self.n_pages, generator=gen)
        at = 0
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n].to(torch.int32)
            at += n
        lens = torch.as_tensor(lens, dtype=torch.int32)
        self.len = (lens if lens.dim() == 3 else (lens[:, None].expand(-1, hkv) if lens.dim() == 1 else lens)[None].expand(layers, -1, -1)).contiguous().clone()
        shape = (layers, self.n_pages, hkv, page, d)
        self.k, self.v = (torch.full(shape, float("nan"), dtype=KIND[dtype]) for _ in range(2))
        for layer in range(layers):
            for b in range(self.batch):
                for h in range(hkv):
                    n = int(self.len[layer, b, h])
                    for pool in (self.k, self.v):
                        rows = torch.randn((held[b] * page, d), generator=gen).to(KIND[dtype])
                        rows[n:] = float("nan")
                        pool[layer, self.table[b, :held[b]].long(), h] = rows.view(held[b], page, d)
        self.pos = torch.full((layers, self.batch, hkv, slots), -77, dtype=torch.int32)
        self.weight = torch.full((layers, self.batch, hkv, slots), float("nan"))
        for layer in range(layers):
            for b in range(self.batch):
                for h in range(hkv):
                    n = int(self.len[layer, b, h])
                    self.pos[layer, b, h, :n] = torch.randperm(3 * n + 1, generator=gen)[:n].to(torch.int32)
                    self.weight[layer, b, h, :n] = torch.rand(n, generator=gen)
        strides = (hkv * page * d, d, hkv * d) if tokens_first else (hkv * page * d, page * d, d)
        self.pages = ckv.Pages(hq, hkv, d, dtype, page, self.n_pages, self.room, *strides, table_pitch=pitch, slot_pitch=slots, softmax_scale=scale)
        self.scale = scale or d ** -0.5

    def pool(self, x):
        """Device pools of the layers."""
        y = (x.transpose(2, 3) if self.tokens_first else x).contiguous().to(DEV)
        return list(y.unbind(0))

    def back(self, pools):
        x = torch.stack(pools).cpu()
        return x.transpose(2, 3).contiguous() if self.tokens_first else x

    def slots(self, b, h, n, layer=0):
        """Indices of the slots whose pages are there, and their places in the pools."""
        s = torch.arange(n)
        page = self.table[b].long()[s // self.page]
        there = (page >= 0) & (page < self.n_pages)
        return s[there], page[there], (s % self.page)[there]

    def rows(self, pool, b, h, n, layer=0):
        s, page, row = self.slots(b, h, n)
        return s, pool[layer, page, h, row].double()


def attention(cache, q, lens, layer=0):
    """[B][Hq][d] output, [B][Hq] log-sum-exp, [B][Hkv][slots] summed weights in float64, and the largest |v| of every kv-head."""
    B, hkv, g, d = cache.batch, cache.hkv, cache.hq // cache.hkv, cache.d
    out, lse = torch.zeros((B, cache.hq, d), dtype=torch.float64), torch.full((B, cache.hq), float("-inf"), dtype=torch.float64)
    weight, top = torch.zeros(cache.weight.shape[1:], dtype=torch.float64), torch.zeros((B, hkv), dtype=torch.float64)
    for b in range(B):
        for h in range(hkv):
            s, k = cache.rows(cache.k, b, h, int(lens[b][h]), layer)
            if len(s) == 0:
                continue
            _, v = cache.rows(cache.v, b, h, int(lens[b][h]), layer)
            heads = slice(h * g, (h + 1) * g)
            x = (q[b, heads].double() @ k.t()) * cache.scale
            lse[b, heads] = torch.logsumexp(x, 1)
            p = torch.exp(x - lse[b, heads, None])
            out[b, heads] = p @ v
            weight[b, h, s] = p.sum(0)
            top[b, h] = v.abs().max()
    return out, lse, weight, top


def same_bits(x, y):
    """Equal bit for bit, NaN included."""
    kind = {1: torch.uint8, 2: torch.int16, 4: torch.int32}[x.element_size()]
    return torch.equal(x.contiguous().view(kind), y.contiguous().view(kind))
