"""chunkkv_rotate against float64 and against the rotation of chunkkv_paged_append; layouts, in place, gradients, graphs."""
import math

import pytest
import torch

import paper_2502_00299_amd as ckv
from tests.rows_helpers import DEV, HALF_STEP, KIND

pytestmark = pytest.mark.gpu
TYPES = [ckv.BF16, ckv.F16, ckv.F32]


def turned(x, positions, freq, interleaved, magnitude):
    """[seqs][tokens][heads][d] in 64 bits, and each element's largest possible sum of terms."""
    y, size, r = x.double().clone(), x.double().abs().clone(), 2 * len(freq)
    a = (positions.double()[..., None] * freq.double())[:, :, None]
    i = torch.arange(r // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + r // 2)
    u, v = y[..., p].clone(), y[..., q].clone()
    y[..., p], y[..., q] = magnitude * (u * a.cos() - v * a.sin()), magnitude * (v * a.cos() + u * a.sin())
    size[..., p] = size[..., q] = magnitude * (u.abs() + v.abs())
    return y, size


def check(got, x, positions, freq, interleaved, magnitude, dtype):
    want, size = turned(x, positions, freq, interleaved, magnitude)
    r = 2 * len(freq)
    # angle: 3 * 2^-25 of a revolution at 2^31, in proportion to the angle's revolutions elsewhere (2^-53 each of product and
    # reduction, three of them); sine and cosine 1.6 * 2^-24 + 2^-24 for the magnitude, product and sum 2^-24 each
    revolutions = (positions.double().abs().amax() if positions.numel() else 0) * float(freq.double().max()) / (2 * math.pi)
    off = 2 * math.pi * 3 * 2.0 ** -53 * revolutions + 5 * 2.0 ** -24
    bound = size * off + (HALF_STEP[dtype] * (1 + off) * want.abs() if dtype != ckv.F32 else 0) + (2.0 ** -25 if dtype == ckv.F16 else 1e-38)
    err = (got.double().cpu() - want).abs()
    assert (err[..., :r] <= bound[..., :r]).all(), float((err[..., :r] / bound[..., :r]).max())
    assert torch.equal(got.cpu()[..., r:], x[..., r:])


def rows(gen, dtype, *shape):
    return torch.randn(shape, generator=gen).to(KIND[dtype])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rotary", [(64, 64), (64, 16), (64, 48), (128, 128), (128, 16), (128, 64), (128, 112)])
@pytest.mark.parametrize("interleaved", [False, True])
def test_parts_and_orders(lib, dtype, d, rotary, interleaved):
    """Views of a fused projection in; queries to rows of their own, keys to a cache [seqs][heads][tokens][d]."""
    gen = torch.Generator().manual_seed(rotary)
    for n, t, hq, hk, magnitude in ((1, 1, 4, 1, 1.0), (3, 37, 7, 2, 1.1386), (2, 5, 32, 8, 0.5)):
        qkv = rows(gen, dtype, n, t, hq + 2 * hk, d)
        q, k = qkv[:, :, :hq], qkv[:, :, hq:hq + hk]
        freq = ckv.chunkkv_rotary_frequencies(rotary, 10000.0, 4.0, 1.0, 32.0, 4096.0)
        pos = torch.randint(-1000, 200000, (n, t), generator=gen, dtype=torch.int32)
        dqkv = qkv.to(DEV)
        q_out = torch.full((n, t, hq, d), 7.0, dtype=KIND[dtype], device=DEV)
        cache = torch.full((n, hk, t + 3, d), 7.0, dtype=KIND[dtype], device=DEV)
        k_out = cache[:, :, 2:-1].transpose(1, 2)
        ckv.chunkkv_rotate(dqkv[:, :, :hq], dqkv[:, :, hq:hq + hk], pos.to(DEV), freq.to(DEV), interleaved, magnitude, q_out, k_out)
        check(q_out, q, pos, freq, interleaved, magnitude, dtype)
        check(k_out, k, pos, freq, interleaved, magnitude, dtype)
        assert (cache[:, :, :2] == 7.0).all() and (cache[:, :, -1] == 7.0).all() and torch.equal(dqkv.cpu(), qkv)
        # each alone, and in place: the same bits, and nothing else touched
        alone = torch.zeros_like(q_out)
        ckv.chunkkv_rotate(dqkv[:, :, :hq], None, pos.to(DEV), freq.to(DEV), interleaved, magnitude, alone, None)
        assert torch.equal(alone, q_out)
        dq, dk = dqkv[:, :, :hq], dqkv[:, :, hq:hq + hk]
        ckv.chunkkv_rotate(None, dk, pos.to(DEV), freq.to(DEV), interleaved, magnitude, None, dk)
        assert torch.equal(dk, k_out) and torch.equal(dq.cpu(), q)
        ckv.chunkkv_rotate(dq, None, pos.to(DEV), freq.to(DEV), interleaved, magnitude, dq, None)
        assert torch.equal(dq, q_out) and torch.equal(dqkv[:, :, hq + hk:].cpu(), qkv[:, :, hq + hk:])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
def test_far_positions(lib, dtype, interleaved):
    gen = torch.Generator().manual_seed(1)
    pos = torch.tensor([0, 1, -1, 1 << 20, 2 ** 31 - 1, -(2 ** 31), 123456789], dtype=torch.int32)
    for d in (64, 128):
        x = rows(gen, dtype, 1, 7, 5, d)
        freq = ckv.chunkkv_rotary_frequencies(d, 500000.0)
        y = torch.zeros_like(x, device=DEV)
        ckv.chunkkv_rotate(x[0].to(DEV), None, pos.to(DEV), freq.to(DEV), interleaved, 1.0, y[0], None)
        check(y, x, pos[None], freq, interleaved, 1.0, dtype)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("rotary", [128, 64])
def test_as_append_rotates(lib, dtype, interleaved, rotary):
    """Tokens on their way into pages and rows anywhere: each within its bound of the exact rotation (a compiler may round a sum and its
    conversion to 16 bits in one step or in two)."""
    gen = torch.Generator().manual_seed(2)
    T, hq, hkv, d = 40, 8, 2, 128
    qkv = rows(gen, dtype, T, hq + 2 * hkv, d).to(DEV)
    q, k, v = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    pos, freq = torch.arange(100000, 100000 + T, dtype=torch.int32, device=DEV), ckv.chunkkv_rotary_frequencies(rotary, 500000.0).to(DEV)
    pages = ckv.Pages(hq, hkv, d, dtype, 16, 4, [T])
    kp, vp = (torch.zeros(4, hkv, 16, d, dtype=KIND[dtype], device=DEV) for _ in range(2))
    table, length = torch.arange(3, dtype=torch.int32, device=DEV)[None], torch.zeros(1, hkv, dtype=torch.int32, device=DEV)
    q_app = torch.zeros(T, hq, d, dtype=KIND[dtype], device=DEV)
    ckv.chunkkv_paged_append(pages, [T], q, k, v, pos, None, None, 0.0, freq, interleaved, q_app, table, kp, vp, length, length, None, None)
    q_out, k_out = torch.zeros_like(q_app), torch.zeros(hkv, 48, d, dtype=KIND[dtype], device=DEV)
    ckv.chunkkv_rotate(q, k, pos, freq, interleaved, 0.0, q_out, k_out.transpose(0, 1)[:T])
    k_app = kp[:3].transpose(0, 1).reshape(hkv, 48, d)
    for x, both in ((q, (q_out, q_app)), (k, (k_out.transpose(0, 1)[:T], k_app.transpose(0, 1)[:T]))):
        for y in both:
            check(y[None], x[None].cpu(), pos[None].cpu(), freq.cpu(), interleaved, 1.0, dtype)
    assert not k_out[:, T:].any() and not k_app[:, T:].any()


@pytest.mark.parametrize("interleaved", [False, True])
def test_gradient_is_the_rotation_back(lib, interleaved):
    """<dL/dy, R x> has the gradient R^T dL/dy: against autograd of the plain formula, and against differences (the map is linear, so the
    difference of any step is the gradient's product with it)."""
    gen = torch.Generator().manual_seed(3)
    d, rotary, magnitude = 64, 48, 1.25
    x, up = torch.randn((2, 9, 3, d), generator=gen), torch.randn((2, 9, 3, d), generator=gen)
    pos, freq = torch.randint(0, 5000, (2, 9), generator=gen, dtype=torch.int32), ckv.chunkkv_rotary_frequencies(rotary, 10000.0)

    def call(y, p):
        out = torch.zeros_like(y, device=DEV)
        ckv.chunkkv_rotate(y.to(DEV), None, p.to(DEV), freq.to(DEV), interleaved, magnitude, out, None)
        return out.double().cpu()

    leaf = x.double().requires_grad_()
    a = (pos.double()[..., None] * freq.double())[:, :, None]
    i = torch.arange(rotary // 2)
    p, q = (2 * i, 2 * i + 1) if interleaved else (i, i + rotary // 2)
    u, v = leaf[..., p], leaf[..., q]
    y = leaf.index_copy(3, torch.cat((p, q)), torch.cat((magnitude * (u * a.cos() - v * a.sin()), magnitude * (v * a.cos() + u * a.sin())), -1))
    y.backward(up.double())
    grad = call(up, -pos)
    # 2 terms of up to |up| * magnitude, each off by 5 * 2^-24 and the angle's share (800 revolutions: 2^-40)
    assert (grad - leaf.grad).abs().max() <= 2 * float(up.abs().max()) * magnitude * 6 * 2.0 ** -24
    step = torch.randn(x.shape, generator=gen)
    change = ((call(x + step, pos) - call(x, pos)) * up.double()).sum()
    n = x.numel()
    assert abs(change - (grad * step.double()).sum()) <= n * 8 * 2.0 ** -24 * 20 * 4


def test_back_and_forth(lib):
    """Keys move from position p to p' by p' - p: as rotated to p' at once, to the roundings of both (fp32: none above 2^-20)."""
    gen = torch.Generator().manual_seed(4)
    x = torch.randn((64, 4, 128), generator=gen).to(DEV)
    freq = ckv.chunkkv_rotary_frequencies(128, 500000.0).to(DEV)
    p, q = torch.arange(64, dtype=torch.int32, device=DEV) + 1000, torch.arange(64, dtype=torch.int32, device=DEV) * 3
    a, b, c = (torch.zeros_like(x) for _ in range(3))
    ckv.chunkkv_rotate(None, x, p, freq, False, 1.0, None, a)
    ckv.chunkkv_rotate(None, a, q - p, freq, False, 1.0, None, b)
    ckv.chunkkv_rotate(None, x, q, freq, False, 1.0, None, c)
    assert (b - c).abs().max() <= 2.0 ** -20 * float(x.abs().max())


@pytest.mark.parametrize("tokens", [1, 63, 1000, 4097, 20000])
@pytest.mark.parametrize("heads", [(1, 0), (0, 3), (32, 8), (129, 7)])
def test_sizes(lib, tokens, heads):
    """How many wavefronts share a token depends on both."""
    gen = torch.Generator(device=DEV).manual_seed(tokens)
    hq, hk = heads
    d = 64
    q, k = (torch.randn((tokens, h, d), generator=gen, device=DEV).bfloat16() if h else None for h in (hq, hk))
    pos, freq = torch.arange(tokens, dtype=torch.int32, device=DEV), ckv.chunkkv_rotary_frequencies(d, 10000.0)
    q_out, k_out = (None if x is None else torch.zeros_like(x) for x in (q, k))
    ckv.chunkkv_rotate(q, k, pos, freq.to(DEV), False, 1.0, q_out, k_out)
    for x, y in ((q, q_out), (k, k_out)):
        if x is not None:
            at = torch.unique(torch.cat((torch.arange(min(tokens, 40)), torch.arange(max(0, tokens - 40), tokens))))
            check(y[at.to(DEV)][None], x[at.to(DEV)][None].cpu(), at.int()[None], freq, False, 1.0, ckv.BF16)
    if tokens == 20000 and hq:   # the rest by a plain pass on the device, in 64 bits
        want, _ = turned(q.cpu()[None], pos.cpu()[None], freq, False, 1.0)
        assert (q_out.cpu()[None].double() - want).abs().max() <= 2.0 ** -8 * float(want.abs().max()) * 1.01


def test_far_rows(lib):
    """Rows past 4 GB of an array, sequences and tokens far apart."""
    d, far = 64, 1 << 28
    x = torch.zeros(9 * far + 64 * 8, dtype=torch.bfloat16, device=DEV)
    y = torch.zeros_like(x)
    v, w = (t.as_strided((2, 3, 2, d), (6 * far, far, d, 1)) for t in (x, y))
    small = torch.randn((2, 3, 2, d)).bfloat16()
    v.copy_(small)
    pos, freq = torch.arange(6, dtype=torch.int32).view(2, 3), ckv.chunkkv_rotary_frequencies(d, 10000.0)
    ckv.chunkkv_rotate(v, None, pos.to(DEV), freq.to(DEV), False, 1.0, w, None)
    check(w, small, pos, freq, False, 1.0, ckv.BF16)


def test_graph(lib):
    x = torch.randn((3, 50, 4, 64), device=DEV).bfloat16()
    pos, freq = torch.arange(150, dtype=torch.int32, device=DEV).view(3, 50), ckv.chunkkv_rotary_frequencies(64, 10000.0).to(DEV)
    y, eager = torch.zeros_like(x), torch.zeros_like(x)
    call = lambda to: ckv.chunkkv_rotate(x, x, pos, freq, True, 1.5, to, torch.zeros_like(x) if to is eager else other)
    other = torch.zeros_like(x)
    call(y)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        call(y)
    for _ in range(3):
        x.normal_()
        pos.add_(7)
        call(eager)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, eager) and torch.equal(other, eager)


def test_refused_and_empty(lib):
    x = torch.zeros((5, 4, 64), dtype=torch.bfloat16, device=DEV)
    y, pos, freq = torch.zeros_like(x), torch.zeros(5, dtype=torch.int32, device=DEV), torch.zeros(32, device=DEV)
    for q, k, p, f, qo, ko in [(x, None, pos, freq, None, None), (x, None, pos, freq, y.float(), None), (x, None, pos, freq, y[:4], None), (x, x[:4], pos, freq, y, y[:4]),
                               (x, None, pos[:4], freq, y, None), (x, None, pos.long(), freq, y, None), (x, None, pos, freq.double(), y, None), (None, None, pos, freq, None, None),
                               (x.double(), None, pos, freq, y.double(), None), (x[..., ::2], None, pos, freq, y[..., ::2], None), (x.cpu(), None, pos, freq, y, None)]:
        with pytest.raises(ValueError):
            ckv.chunkkv_rotate(q, k, p, f, False, 1.0, qo, ko)
    for f, m, status in [(torch.zeros(64, device=DEV), 1.0, 2), (torch.zeros(4, device=DEV), 1.0, 3), (freq, -1.0, 2), (freq, math.inf, 2), (None, 1.0, 2)]:
        with pytest.raises(ckv.ChunkKVError) as e:
            ckv.chunkkv_rotate(x, None, pos, f, False, m, y, None)
        assert e.value.status == status
    with pytest.raises(ckv.ChunkKVError):   # in place, to other places
        ckv.chunkkv_rotate(x[:4], None, pos, freq, False, 1.0, x.view(-1).as_strided((4, 4, 64), (64, 256, 1)), None)
    empty = x[:0]
    ckv.chunkkv_rotate(empty, None, pos, freq, False, 1.0, empty, None)
    ckv.chunkkv_rotate(x.view(0 + 1, 5, 4, 64)[:0], None, pos, freq, False, 1.0, y.view(1, 5, 4, 64)[:0], None)
