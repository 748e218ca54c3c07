"""Head norms, rotation and storing of new tokens, against float64."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from oracle import paged_oracle as orc
from tests import paged_helpers as H

pytestmark = pytest.mark.gpu
DEV = H.DEV
F32, BF16, F16 = ckv.F32, ckv.BF16, ckv.F16


def turned(x, norm, eps, positions, freq, interleaved):
    """[T][heads][d] in float64, and the magnitudes that its rounding errors go by."""
    y = x.double()
    if norm is not None:
        y = y / torch.sqrt((y * y).mean(-1, keepdim=True) + eps) * norm.double()
    size = y.abs().clone()
    if freq is not None:
        half = len(freq)
        i = torch.arange(half)
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        angle = torch.remainder(positions.double()[:, None, None] * freq.double(), 2 * torch.pi)
        c, s = torch.cos(angle), torch.sin(angle)
        p, q = y[..., a], y[..., b]
        y = y.clone()
        y[..., a], y[..., b] = p * c - q * s, q * c + p * s
        size[..., a] = size[..., b] = p.abs() + q.abs()
    return y, size


def close(got, want, size, dtype):
    # fp32: a norm's sum of squares 16 roundings, its root, quotient and products 5; sine and cosine 4 of a unit (argument and
    # value), the rotation 3: 28 * 2^-24 of the pair's magnitudes; then half a step of the type (of fp16's least step, 2^-24)
    bound = 28 * 2.0 ** -24 * size + (H.HALF_STEP[dtype] * want.abs() * 1.001 if dtype != F32 else 0.0) + (2.0 ** -25 if dtype == F16 else 1e-37)
    return bool(((got.double() - want).abs() <= bound).all())


def prepared(gen, dtype, hq, hkv, d, new, norm, rotary, positions=None):
    T = sum(new)
    qkv = torch.randn((T, hq + 2 * hkv, d), generator=gen).to(H.KIND[dtype])
    pos = torch.randint(0, 300000, (T,), generator=gen).to(torch.int32) if positions is None else positions
    qn, kn = ((1 + 0.3 * torch.randn(d, generator=gen)).to(H.KIND[dtype]) if norm else None for _ in range(2))
    freq = (10000.0 ** (-torch.arange(0, rotary, 2, dtype=torch.float64) / rotary)).float() if rotary else None
    return qkv, pos, qn, kn, freq


def call(cache, new, qkv, pos, qn, kn, freq, inter, kp, vp, length, length_out, token_pos, weight, eps=1e-5, with_q=True, stream=None):
    hq, hkv = cache.hq, cache.hkv
    dev = qkv.to(DEV)
    q_out = torch.full((sum(new), hq, cache.d), float("nan"), dtype=H.KIND[cache.dtype], device=DEV) if with_q else None
    up = lambda x: None if x is None else x.to(DEV)  # noqa: E731
    ckv.chunkkv_paged_append(cache.pages, new, dev[:, :hq] if with_q else None, dev[:, hq:hq + hkv], dev[:, hq + hkv:], up(pos), up(qn) if with_q else None, up(kn), eps,
                             up(freq), inter, q_out, up(cache.table), kp, vp, length, length_out, token_pos, weight, stream)
    return q_out


@pytest.mark.parametrize("norm,rotary,inter", [(True, 1, False), (True, 1, True), (False, 1, False), (True, 0, False), (False, 0, False), (True, 16, False), (False, 32, True),
                                               (True, 48, False)])
@pytest.mark.parametrize("dtype,hq,hkv,d", [(BF16, 8, 2, 128), (F16, 7, 1, 64), (F32, 4, 4, 128), (F32, 6, 3, 64), (BF16, 5, 5, 64), (F16, 40, 8, 128)])
def test_against_float64(lib, dtype, hq, hkv, d, norm, rotary, inter):
    """New tokens of several sequences, none of one, past the room of another; both layouts; slots elsewhere stay as they are."""
    rotary = d if rotary == 1 else rotary
    gen = torch.Generator().manual_seed(d + hq + rotary)
    new, lens, room = [3, 0, 1, 40, 7], [0, 5, 15, 30, 20], [3, 5, 16, 100, 22]
    for first, in_place in ((False, False), (True, True)):
        cache = H.Cache(gen, dtype, hq, hkv, d, 16 if first else 48, room, lens, tokens_first=first)
        cache.len[0, 3] -= torch.arange(hkv, dtype=torch.int32)         # heads of different length
        qkv, pos, qn, kn, freq = prepared(gen, dtype, hq, hkv, d, new, norm, rotary)
        kp, vp = cache.pool(cache.k)[0], cache.pool(cache.v)[0]
        length = cache.len[0].to(DEV)
        after = length if in_place else torch.full_like(length, -9)
        tp, tw = cache.pos[0].to(DEV), cache.weight[0].to(DEV)
        q_out = call(cache, new, qkv, pos, qn, kn, freq, inter, kp, vp, length, after, tp, tw)
        want_q, size = turned(qkv[:, :hq], qn, 1e-5, pos, freq, inter)
        assert close(q_out.cpu(), want_q, size, dtype)
        if not norm and not rotary:
            assert H.same_bits(q_out.cpu(), qkv[:, :hq])
        want_k, size_k = turned(qkv[:, hq:hq + hkv], kn, 1e-5, pos, freq, inter)
        pool_k, pool_v = cache.k.clone(), cache.v.clone()
        want_pos, want_weight, want_len = cache.pos[0].clone(), cache.weight[0].clone(), cache.len[0].clone()
        got_k, got_v = cache.back([kp]), cache.back([vp])
        at = 0
        for b, n in enumerate(new):
            for h in range(hkv):
                for i in range(n):
                    slot = int(cache.len[0, b, h]) + i
                    if slot >= room[b]:
                        continue
                    page, row = int(cache.table[b, slot // cache.page]), slot % cache.page
                    assert close(got_k[0, page, h, row], want_k[at + i, h], size_k[at + i, h], dtype)
                    pool_k[0, page, h, row] = got_k[0, page, h, row]
                    pool_v[0, page, h, row] = qkv[at + i, hq + hkv + h]
                    want_pos[b, h, slot], want_weight[b, h, slot] = pos[at + i], 0.0
                want_len[b, h] = min(room[b], int(cache.len[0, b, h]) + n)
            at += n
        assert H.same_bits(got_k, pool_k) and H.same_bits(got_v, pool_v)
        assert torch.equal(tp.cpu(), want_pos) and H.same_bits(tw.cpu(), want_weight) and torch.equal(after.cpu(), want_len)


def test_one_row_against_the_oracle(lib):
    """The oracle states the formula element by element; here the two meet."""
    gen = torch.Generator().manual_seed(3)
    cache = H.Cache(gen, F32, 2, 1, 64, 16, [2], [0])
    for inter in (False, True):
        qkv, pos, qn, kn, freq = prepared(gen, F32, 2, 1, 64, [2], True, 32, torch.tensor([7, 123456], dtype=torch.int32))
        out = call(cache, [2], qkv, pos, qn, kn, freq, inter, cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV), cache.len[0].to(DEV), None, None).cpu()
        for t in range(2):
            for h in range(2):
                want = torch.from_numpy(orc.norm_and_rotate(qkv[t, h].numpy(), qn.numpy(), 1e-5, int(pos[t]), freq.double().numpy(), inter))
                assert float((out[t, h].double() - want).abs().max()) <= 28 * 2.0 ** -24 * 2 * float(qkv.abs().max()) * 2


@pytest.mark.parametrize("position", [0, 1, -1, 2 ** 20 + 1, 2 ** 31 - 1, -(2 ** 31)])
def test_far_positions(lib, position):
    """Angles of far positions: 31 bits times 24 bits do not fit a double's 53 by two; product, division and its constant leave
    3 * 2^-25 of a revolution at 2^31."""
    gen = torch.Generator().manual_seed(8)
    cache = H.Cache(gen, F32, 4, 1, 128, 16, [1], [0])
    qkv, pos, qn, kn, freq = prepared(gen, F32, 4, 1, 128, [1], False, 128, torch.tensor([position], dtype=torch.int32))
    out = call(cache, [1], qkv, pos, None, None, freq, False, cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV), cache.len[0].to(DEV), None, None)
    i = torch.arange(64)
    rev = [(position * int(f * 2.0 ** 40)) for f in freq.double().tolist()]                     # inv_freq >= 2^-14 has 24 bits: exact
    assert all(float(f) * 2.0 ** 40 == int(float(f) * 2.0 ** 40) for f in freq.double().tolist())
    import math
    from fractions import Fraction
    turn = Fraction(31415926535897932384626433832795028841971693993751, 10 ** 49) * 2
    angle = torch.tensor([float(Fraction(r, 2 ** 40) % turn) for r in rev], dtype=torch.float64)
    x = qkv[0, :4].double()
    want = torch.cat((x[:, i] * torch.cos(angle) - x[:, i + 64] * torch.sin(angle), x[:, i + 64] * torch.cos(angle) + x[:, i] * torch.sin(angle)), 1)
    size = x[:, i].abs() + x[:, i + 64].abs()
    bound = (28 * 2.0 ** -24 + 2 * math.pi * 3 * 2.0 ** -25 * (abs(position) / 2.0 ** 31)) * torch.cat((size, size), 1)
    assert bool(((out.cpu()[0].double() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype,batch,new", [(BF16, 150, 1), (F16, 131, 2), (BF16, 1, 2000), (F32, 3, 500)])
def test_many(lib, dtype, batch, new):
    """More sequences than a launch's tables hold, prompts: against the same tokens one sequence at a time, to the bit."""
    gen = torch.Generator().manual_seed(batch)
    news = [new] * batch
    if batch > 100:
        news[5], news[128] = 0, 9
    lens = [(11 * i) % 40 for i in range(batch)]
    room = [n + m for n, m in zip(lens, news)]
    cache = H.Cache(gen, dtype, 8, 2, 128, 16, room, lens)
    qkv, pos, qn, kn, freq = prepared(gen, dtype, 8, 2, 128, news, True, 128)
    kp, vp, length = cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV)
    out = call(cache, news, qkv, pos, qn, kn, freq, False, kp, vp, length, length, None, None)
    want, size = turned(qkv[:, :8], qn, 1e-5, pos, freq, False)
    assert close(out.cpu(), want, size, dtype)
    assert length.cpu().tolist() == [[n] * 2 for n in room]
    got_k, got_v = cache.back([kp])[0], cache.back([vp])[0]
    want_k, size_k = turned(qkv[:, 8:10], kn, 1e-5, pos, freq, False)
    at = 0
    for b, n in enumerate(news):
        s = lens[b] + torch.arange(n)
        page, row = cache.table[b].long()[s // 16], s % 16
        assert close(got_k[page, :, row], want_k[at:at + n], size_k[at:at + n], dtype)
        assert H.same_bits(got_v[page, :, row], qkv[at:at + n, 10:])
        at += n


def test_pages_that_are_not_there_and_keys_alone(lib):
    """Nothing is stored for them, positions and lengths are kept all the same; without queries only keys and values."""
    gen = torch.Generator().manual_seed(2)
    cache = H.Cache(gen, BF16, 4, 2, 64, 16, [40, 40], [10, 10])
    cache.table[0, 1] = -1
    cache.table[1, 1] = cache.n_pages
    qkv, pos, qn, kn, freq = prepared(gen, BF16, 4, 2, 64, [20, 20], True, 64)
    kp, vp, length = cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV)
    tp = cache.pos[0].to(DEV)
    assert call(cache, [20, 20], qkv, pos, qn, kn, freq, False, kp, vp, length, length, tp, None, with_q=False) is None
    assert (length == 30).all() and torch.equal(tp[0, 1, 10:30].cpu(), pos[:20])
    got = cache.back([vp])[0]
    for b in range(2):
        page = int(cache.table[b, 0])
        assert H.same_bits(got[page, :, 10:].transpose(0, 1), qkv[20 * b:20 * b + 6, 6:])
        got[page] = cache.v[0, page]
    assert H.same_bits(got, cache.v[0])                    # no other page was written


def test_refused_by_the_binding(lib):
    gen = torch.Generator().manual_seed(2)
    cache = H.Cache(gen, BF16, 4, 2, 64, 16, [40], [10])
    qkv, pos, qn, kn, freq = prepared(gen, BF16, 4, 2, 64, [3], True, 64)
    kp, vp, n = cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV)
    good = dict(new=[3], qkv=qkv, pos=pos, qn=qn, kn=kn, freq=freq, inter=False, kp=kp, vp=vp, length=n, length_out=n, token_pos=None, weight=None)
    call(cache, **good)
    for bad in (dict(new=[4]), dict(new=[1, 2]), dict(qkv=qkv.float()), dict(pos=pos[:2]), dict(pos=pos.long()), dict(qn=qn[:32]), dict(freq=torch.ones(12)), dict(kp=kp[:-1].clone()),
                dict(vp=vp.half()), dict(length=n[:, :1].contiguous()), dict(token_pos=cache.pos[0, :, :1].contiguous().to(DEV)), dict(token_pos=cache.pos[0])):
        with pytest.raises((ValueError, ckv.ChunkKVError)):
            call(cache, **{**good, **bad})


def test_no_new_tokens(lib):
    """A step in which no sequence has a token: lengths are carried over, nothing else is touched."""
    gen = torch.Generator().manual_seed(3)
    cache = H.Cache(gen, F16, 4, 2, 64, 16, [40, 9], [10, 9])
    none = torch.zeros((0, 8, 64), dtype=torch.float16)
    kp, vp, n, after = cache.pool(cache.k)[0], cache.pool(cache.v)[0], cache.len[0].to(DEV), torch.full((2, 2), -3, dtype=torch.int32, device=DEV)
    tp = cache.pos[0].to(DEV)
    call(cache, [0, 0], none, torch.zeros(0, dtype=torch.int32), None, None, None, False, kp, vp, n, after, tp, None)
    assert torch.equal(after, n) and H.same_bits(cache.back([kp])[0], cache.k[0]) and H.same_bits(tp.cpu(), cache.pos[0])
    call(cache, [0, 0], none, torch.zeros(0, dtype=torch.int32), None, None, None, False, kp, vp, n, n, None, None)
    assert torch.equal(after, n)
