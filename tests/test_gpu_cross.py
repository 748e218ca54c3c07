"""chunkkv_cross_attention against float64: lengths, layouts, masks, strides, types; graphs and streams."""
import math

import pytest
import torch

import paper_2502_00299_amd as ckv
from tests.rows_helpers import DEV, KIND, attend, near, near_lse

pytestmark = pytest.mark.gpu
NAN = float("nan")


class Job:
    """Host tensors of a call, their device copies, and what the call has to give."""

    def __init__(self, seed, dtype, hq, hkv, d, q_len, states, layout="packed", fused=False, heads_out=False, lens=None, mask=None, scale=0.0, strength=1.0, pad=0):
        gen = torch.Generator().manual_seed(seed)
        self.dtype, self.hq, self.hkv, self.d, self.q_len, self.states, self.scale = dtype, hq, hkv, d, list(q_len), list(states), scale
        B, T, kind = len(q_len), sum(q_len), KIND[dtype]
        self.B, self.T = B, T
        width = hq + 2 * hkv if fused else hq
        self.q_all = (torch.randn((max(T, 1), width, d), generator=gen) * strength).to(kind)
        self.q = self.q_all[:T, :hq]
        most = max([1] + self.states) + pad
        if layout == "packed":       # [sum][hkv][d]
            self.base, run = [], 0
            for n in self.states:
                self.base.append(run * hkv * d)
                run += n
            size, self.sh, self.st = max(run, 1) * hkv * d, d, hkv * d
        elif layout == "padded":     # [B][most][hkv][d]
            self.base, size, self.sh, self.st = [b * most * hkv * d for b in range(B)], B * most * hkv * d, d, hkv * d
        else:                        # [B][hkv][most][d]
            self.base, size, self.sh, self.st = [b * most * hkv * d for b in range(B)], B * most * hkv * d, most * d, d
        self.k, self.v = (torch.full((size,), NAN, dtype=kind) for _ in range(2))
        self.lens = None if lens is None else torch.as_tensor(lens, dtype=torch.int32)
        self.mask = None if mask is None else mask(gen, B, most)
        self.rows = {}
        for b in range(B):
            for h in range(hkv):
                n = self.states[b] if self.lens is None else min(max(int(self.lens[b, h]), 0), self.states[b])
                here = torch.arange(n)
                if self.mask is not None:
                    here = here[self.mask[b, :n] != 0]
                at = self.base[b] + h * self.sh + here * self.st
                at = (at[:, None] + torch.arange(d)).flatten()
                rows = []
                for x in (self.k, self.v):
                    y = (torch.randn((len(here), d), generator=gen) * (strength if x is self.k else 1.0)).to(kind)
                    x[at] = y.flatten()
                    rows.append(y.double())
                self.rows[b, h] = rows
        kw = {}
        if fused:
            kw.update(q_base=[width * d * sum(self.q_len[:b]) for b in range(B)], q_stride_head=d, q_stride_tok=width * d)
        self.heads_out = heads_out
        if heads_out:                # outputs [hq][T][d]
            kw.update(out_base=[d * sum(self.q_len[:b]) for b in range(B)], out_stride_head=max(T, 1) * d, out_stride_tok=d)
        self.plan = ckv.Cross(hq, hkv, d, dtype, self.q_len, self.states, self.base, self.sh, self.st, mask_pitch=most if self.mask is not None else 0, softmax_scale=scale, **kw)

    def want(self):
        g, s = self.hq // self.hkv, self.scale or self.d ** -0.5
        out, bound = (torch.zeros((self.T, self.hq, self.d), dtype=torch.float64) for _ in range(2))
        lse, lbound = (torch.zeros((self.T, self.hq), dtype=torch.float64) for _ in range(2))
        t = 0
        for b, n in enumerate(self.q_len):
            for h in range(self.hkv):
                heads = slice(h * g, (h + 1) * g)
                got = attend(self.q[t:t + n, heads].double().flatten(0, 1), *self.rows[b, h], s, self.dtype)
                for to, x in zip((out, lse, bound, lbound), got):
                    to[t:t + n, heads] = x.view(n, g, *x.shape[1:])
            t += n
        return out, lse, bound, lbound

    def device(self):
        self.dq, self.dk, self.dv = (x.to(DEV) for x in (self.q_all, self.k, self.v))
        self.dlen = None if self.lens is None else self.lens.to(DEV)
        self.dmask = None if self.mask is None else self.mask.to(DEV)
        shape = (self.hq, max(self.T, 1), self.d) if self.heads_out else (max(self.T, 1), self.hq, self.d)
        n = shape[0] * shape[1] * shape[2]
        self.guarded = torch.full((n + 512,), 7.0, dtype=KIND[self.dtype], device=DEV)
        self.out = self.guarded[256:256 + n].view(shape)
        self.lse = torch.full((max(self.T, 1), self.hq), 5.0, device=DEV)
        self.ws = torch.full((ckv.chunkkv_cross_workspace_bytes(self.plan),), 255, dtype=torch.uint8, device=DEV)
        return self

    def call(self, lse=True, stream=None):
        ckv.chunkkv_cross_attention(self.plan, self.dlen, self.dmask, self.dq, self.dk, self.dv, self.out, self.lse if lse else None, self.ws, stream=stream)

    def result(self):
        return (self.out.transpose(0, 1) if self.heads_out else self.out)[:self.T]

    def check(self, what=""):
        out, lse, bound, lbound = self.want()
        self.device()
        self.call(lse=False)
        torch.cuda.synchronize()
        near(self.result(), out, bound, f"out {what}")
        assert (self.lse == 5.0).all()
        self.guarded.fill_(7.0)
        self.call()
        torch.cuda.synchronize()
        near(self.result(), out, bound, f"out beside lse {what}")
        near_lse(self.lse[:self.T], lse, lbound, f"lse {what}")
        assert (self.guarded[:256] == 7.0).all() and (self.guarded[-256:] == 7.0).all()
        first = self.result().clone(), self.lse.clone()
        self.ws.random_(0, 256)
        self.call()
        torch.cuda.synchronize()
        assert torch.equal(first[0], self.result()) and torch.equal(first[1], self.lse), "the same call, other bits"


TYPES = [ckv.BF16, ckv.F16, ckv.F32]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("states", [1, 31, 32, 33, 63, 64, 65, 127, 129, 500])
def test_lengths(lib, dtype, d, states):
    for q_len in (1, 5, 17, 33):
        Job(states, dtype, 8, 2, d, [q_len], [states], layout="heads").check(f"{q_len} over {states}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows", [(1, 1, 63), (1, 1, 64), (1, 1, 65), (7, 1, 9), (7, 1, 10), (4, 1, 16), (4, 2, 32), (4, 1, 33), (16, 1, 17), (256, 1, 1), (96, 3, 7), (5, 5, 300)])
def test_query_rows(lib, dtype, rows):
    """Both sides of the rows that a workgroup has, many heads of a kv-head, many tokens of one."""
    g, hkv, n = rows
    if g > 64:
        g //= hkv
    Job(sum(rows), dtype, g * hkv, hkv, 64, [n], [200], layout="packed").check(str(rows))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["packed", "padded", "heads"])
def test_ragged(lib, dtype, layout):
    """Sequences without queries or states among others, of one token and of one state; rows of a fused projection, outputs by head."""
    q_len, states = [3, 0, 40, 1, 9, 1, 130], [70, 33, 0, 1, 700, 64, 257]
    Job(1, dtype, 12, 3, 128, q_len, states, layout=layout).check()
    Job(2, dtype, 12, 3, 64, q_len, states, layout=layout, fused=True, heads_out=True, pad=0 if layout == "packed" else 5).check()


def test_more_sequences_than_a_launch_has(lib):
    for n in (32, 33, 100):
        Job(n, ckv.BF16, 4, 2, 64, [(i * 5) % 9 for i in range(n)], [(i * 37) % 150 for i in range(n)]).check(str(n))


@pytest.mark.parametrize("dtype", TYPES)
def test_ranges(lib, dtype):
    """Long sequences of few rows, cut into ranges and joined: beside short ones, of one workgroup's rows and of several."""
    Job(3, dtype, 4, 1, 128, [1, 2], [9001, 130], layout="heads").check()
    Job(4, dtype, 8, 2, 64, [70, 1], [4097, 20000], layout="heads").check()
    Job(5, dtype, 8, 2, 64, [1], [65], layout="heads").check()


def random_mask(share):
    return lambda gen, B, n: torch.rand((B, n), generator=gen) >= share


def edges_mask(gen, B, n):
    m = torch.zeros((B, n), dtype=torch.uint8)
    for b in range(B):   # none; the first; the last; a whole tile in the middle; one bit in each tile, as large numbers
        if b % 5 == 1:
            m[b, 0] = 1
        elif b % 5 == 2:
            m[b, n - 1] = 255
        elif b % 5 == 3:
            m[b, 64:128] = 128
        elif b % 5 == 4:
            m[b, 13::64] = 2
    return m


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [random_mask(0.1), random_mask(0.97), random_mask(0.0), edges_mask], ids=["holes", "few", "all", "edges"])
def test_masks(lib, dtype, d, mask):
    """Rows of K and V that the mask takes out are NaN; rows of the mask that leave nothing."""
    Job(6, dtype, 6, 2, d, [3, 50, 1, 30, 2], [300] * 5, layout="padded", mask=mask).check()
    Job(7, dtype, 2, 2, d, [1, 70], [5000, 777], layout="heads", mask=mask).check()


def test_masked_infinities(lib):
    job = Job(8, ckv.F16, 4, 2, 64, [9, 70], [200, 333], layout="padded", mask=random_mask(0.3))
    bad = job.k.isnan()
    for x, y in ((job.k, math.inf), (job.v, -math.inf)):
        x[bad] = y
    job.check()


@pytest.mark.parametrize("dtype", TYPES)
def test_device_lengths(lib, dtype):
    """Heads of other lengths than the sequence, below zero and above it; with a mask too."""
    lens = [[0, 64, 300], [-5, 299, 1], [1000, 65, 128]]
    Job(9, dtype, 6, 3, 64, [2, 70, 33], [300] * 3, layout="heads", lens=lens).check()
    Job(10, dtype, 6, 3, 128, [2, 70, 33], [300] * 3, layout="padded", lens=lens, mask=random_mask(0.4)).check()
    Job(11, dtype, 4, 1, 64, [1], [50000], layout="heads", lens=[[77]]).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("scale", [1e-45, 1e-3, 1.0, 30.0])
def test_scales(lib, dtype, scale):
    Job(12, dtype, 4, 2, 64, [5, 40], [333, 150], scale=scale).check()


@pytest.mark.parametrize("dtype", [ckv.BF16, ckv.F32])
@pytest.mark.parametrize("power", [1e18, 2.2e19])
def test_scores_up_to_the_ends_of_fp32(lib, dtype, power):
    """One key has all the weight: q . k up to 1e38, where the scores in log2 units are none.  Its value is the output, bit by bit."""
    d, n = 64, 300
    gen = torch.Generator().manual_seed(1)
    k = torch.zeros(n, d)
    k[:, 0] = -torch.rand(n, generator=gen) * power * 0.5 - power * 0.1
    k[170, 0] = -power * 0.01
    v = torch.randn((n, d), generator=gen).to(KIND[dtype])
    q = torch.zeros(40, 1, d)
    q[:, 0, 0] = power
    out, lse = torch.zeros((40, 1, d), dtype=KIND[dtype], device=DEV), torch.zeros((40, 1), device=DEV)
    for scale in (0.0, 1.0, 1e-20):
        plan = ckv.Cross(1, 1, d, dtype, [40], [n], [0], d, d, softmax_scale=scale)
        ws = torch.empty(ckv.chunkkv_cross_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
        ckv.chunkkv_cross_attention(plan, None, None, q.to(KIND[dtype]).to(DEV), k.to(KIND[dtype]).to(DEV), v.to(DEV), out, lse, ws)
        assert torch.equal(out.cpu(), v[170].expand(40, 1, d)), scale
        x = float(q[0, 0, 0].to(KIND[dtype])) * float(k[170, 0].to(KIND[dtype])) * (scale or 0.125)
        assert ((lse.double().cpu() - x).abs() <= 2 ** -22 * abs(x)).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_uneven_scores(lib, dtype):
    """Scores that grow along the keys, so that references move in every tile, and fall; equal values come out as they are."""
    for rising in (1, -1):
        job = Job(13, dtype, 4, 1, 64, [3, 30], [700, 700], layout="heads")
        for b in range(2):
            k = job.rows[b, 0][0]
            k[:, 0] = rising * torch.arange(len(k), dtype=torch.float64) / 8
            k.copy_(k.to(KIND[dtype]).double())
            job.k[job.base[b]:job.base[b] + len(k) * 64] = k.to(KIND[dtype]).flatten()
        job.q_all[:, :, 0] = 8.0
        job.check(str(rising))
    job = Job(14, dtype, 4, 1, 64, [3, 30], [700, 555], layout="heads")
    job.v.fill_(1.0 / 3)
    job.device().call()
    if dtype == ckv.F32:   # no output of fewer bits to round to: a sum of n products and one of n weights, as many roundings each as attend() counts
        off = 2 * (700 / 16 + 40) * 2.0 ** -24 * float(job.v[0])
        assert (job.result() - float(job.v[0])).abs().max() <= off
    else:
        assert torch.equal(job.result().cpu(), job.v[0].expand_as(job.result()))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d,rows", [(64, 3), (64, 150), (64, 600), (128, 150), (128, 600)])
def test_references(lib, dtype, d, rows):
    """Tiles whose weights add up to just what a reference stands, a little less and a little more, and single weights at the end of fp16."""
    job = Job(15, dtype, 2, 2, d, [rows], [13 * 64], layout="heads", scale=math.log(2.0))
    level = torch.zeros(13, 64, dtype=torch.float64)
    level[1, 5] = level[2, 40] = 7.0     # one weight of 2^7, in fp16's scale 2^16; in tile 1 it is 2^(15.9995), which rounds to the largest number
    for tile, x in ((3, 9.875), (4, 10.0), (5, 11.0), (6, 14.0), (7, 12.0), (8, -20.0), (9, 30.0), (10, 31.0), (11, 38.0), (12, 38.0)):
        level[tile] = x
    level[12, ::2] = -1000.0
    k = torch.zeros(13 * 64, d, dtype=torch.float64)
    k[:, 0] = level.flatten()
    k[64 + 5, 1] = 1.0
    k = k.to(KIND[dtype])
    for h in range(2):
        job.rows[0, h][0] = k.double()
        at = job.base[0] + h * job.sh
        job.k[at:at + k.numel()] = k.flatten()
    job.q_all.zero_()
    job.q_all[:, :, 0] = torch.tensor([1.0, 0.5, 2.0, -1.0, 0.0]).to(KIND[dtype])[torch.arange(rows) % 5][:, None]
    job.q_all[:, 0, 1] = -0.0005         # 65513: to 65504
    job.q_all[:, 1, 1] = -0.0002         # 65527: beyond it
    job.check()


def test_far_offsets(lib):
    """States, queries and outputs behind the first 4 GB of their arrays, keys 64 KB apart so that a sequence's span passes 32 bits."""
    d, hkv, n, far = 64, 2, 70000, 1 << 15
    k = torch.zeros(n * far + hkv * d, dtype=torch.bfloat16, device=DEV)
    gen = torch.Generator().manual_seed(2)
    small = torch.randn((n, hkv, d), generator=gen).bfloat16()
    k.as_strided((n, hkv, d), (far, d, 1)).copy_(small.to(DEV))
    q = torch.randn((33, 4, d), generator=gen).bfloat16()
    plan = ckv.Cross(4, hkv, d, ckv.BF16, [33], [n], [0], d, far)
    near_plan = ckv.Cross(4, hkv, d, ckv.BF16, [33], [n], [0], d, hkv * d)
    outs = []
    for p, x in ((plan, k), (near_plan, small.to(DEV))):
        out = torch.zeros((33, 4, d), dtype=torch.bfloat16, device=DEV)
        ws = torch.empty(ckv.chunkkv_cross_workspace_bytes(p), dtype=torch.uint8, device=DEV)
        ckv.chunkkv_cross_attention(p, None, None, q.to(DEV), x, x, out, None, ws)
        outs.append(out.cpu())
    assert torch.equal(*outs)
    # queries and outputs at the end of the same array's size
    at = (n * far) // 128 * 128 - 64 * 4 * d
    big = torch.zeros(n * far + hkv * d, dtype=torch.bfloat16, device=DEV)
    big[at:at + 33 * 4 * d] = q.to(DEV).flatten()
    plan = ckv.Cross(4, hkv, d, ckv.BF16, [33], [n], [0], d, far, q_base=[at], q_stride_head=d, q_stride_tok=4 * d, out_base=[at], out_stride_head=d, out_stride_tok=4 * d)
    out = torch.zeros_like(big)
    ckv.chunkkv_cross_attention(plan, None, None, big, k, k, out, None, torch.empty(ckv.chunkkv_cross_workspace_bytes(plan), dtype=torch.uint8, device=DEV))
    assert torch.equal(out[at:at + 33 * 4 * d].view(33, 4, d).cpu(), outs[0]) and not out[:at].any()


def test_long_cache(lib):
    """A million states and more, one of them with all the weight, wherever it is."""
    d, n = 64, (1 << 20) + 77
    k = torch.zeros((n, d), dtype=torch.float16, device=DEV)
    v = torch.zeros_like(k)
    v[:, 0] = 1.0
    for place in (0, 123456, n - 1):
        k[place, 0], v[place, 1] = 100.0, 2.0
        q = torch.zeros((3, 2, d), dtype=torch.float16, device=DEV)
        q[:, :, 0] = 10.0
        plan = ckv.Cross(2, 1, d, ckv.F16, [3], [n], [0], d, d)
        out = torch.zeros_like(q)
        ckv.chunkkv_cross_attention(plan, None, None, q, k, v, out, None, torch.empty(ckv.chunkkv_cross_workspace_bytes(plan), dtype=torch.uint8, device=DEV))
        assert (out[..., 0] == 1.0).all() and (out[..., 1] == 2.0).all() and not out[..., 2:].any()
        k[place, 0], v[place, 1] = 0.0, 0.0
    plan.softmax_scale = 1e-45   # all the same weight
    out.zero_()
    ckv.chunkkv_cross_attention(plan, None, None, q, k, v, out, None, torch.empty(ckv.chunkkv_cross_workspace_bytes(plan), dtype=torch.uint8, device=DEV))
    assert (out[..., 0] == 1.0).all()


def test_graphs_and_streams(lib):
    """Two captured calls that share a workspace, replayed in turn on new inputs; eager calls on two streams with workspaces of their own."""
    jobs = [Job(20, ckv.BF16, 8, 2, 128, [3, 1], [3000, 40], layout="heads").device(), Job(21, ckv.F16, 4, 4, 64, [70], [900], layout="heads", mask=random_mask(0.2)).device()]
    ws = max((j.ws for j in jobs), key=lambda x: x.numel())
    for j in jobs:
        j.ws = ws
        j.call()
    torch.cuda.synchronize()
    graphs = []
    for j in jobs:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            j.call()
        graphs.append(g)
    for turn in range(4):
        for j, g in zip(jobs, graphs):
            j.dq.normal_()
            j.call()
            torch.cuda.synchronize()
            eager = j.out.clone(), j.lse.clone()
            j.out.zero_()
            j.lse.zero_()
            ws.random_(0, 256)
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(j.out, eager[0]) and torch.equal(j.lse, eager[1]), turn
    streams = [torch.cuda.Stream() for _ in jobs]
    for j in jobs:
        j.call()
        j.kept = j.out.clone()
        j.out.zero_()
        j.ws = torch.empty(ckv.chunkkv_cross_workspace_bytes(j.plan), dtype=torch.uint8, device=DEV)
    torch.cuda.synchronize()
    for _ in range(3):
        for j, s in zip(jobs, streams):
            j.call(stream=s)
    torch.cuda.synchronize()
    for j in jobs:
        assert torch.equal(j.out, j.kept)


def test_nothing_to_do(lib):
    plan = ckv.Cross(4, 2, 64, ckv.BF16, [0, 0], [100, 0], [0, 0], 64, 128)
    ckv.chunkkv_cross_attention(plan, None, None, None, None, None, None, None, None)
    out = torch.full((5, 4, 64), 3.0, dtype=torch.bfloat16, device=DEV)
    lse = torch.zeros((5, 4), device=DEV)
    plan = ckv.Cross(4, 2, 64, ckv.BF16, [2, 3], [0, 0], [0, 0], 64, 128)
    ckv.chunkkv_cross_attention(plan, None, None, torch.zeros_like(out), None, None, out, lse, None)
    assert not out.any() and (lse == -math.inf).all()


def test_sizes_and_types_that_are_refused(lib):
    job = Job(22, ckv.BF16, 4, 2, 64, [5], [300], layout="heads", mask=random_mask(0.1)).device()
    good = dict(dq=job.dq, dk=job.dk, dv=job.dv, out=job.out, lse=job.lse, dmask=job.dmask, ws=job.ws)
    for name, bad in [("dq", job.dq.float()), ("dq", job.dq[:4].clone()), ("dk", job.dk[:-64].clone()), ("dv", job.dv.half()), ("out", job.guarded[:4 * 4 * 64].clone()), ("lse", job.lse[:4]), ("lse", job.lse.double()),
                      ("dmask", job.dmask.int()), ("dmask", job.dmask[:, :-1]), ("dk", job.dk.cpu())]:
        setattr(job, name, bad)
        with pytest.raises(ValueError):
            job.call()
        setattr(job, name, good[name])
    job.plan = ckv.Cross(4, 2, 64, ckv.BF16, [5], [30000], [0], 30000 * 64, 64)
    job.dk = job.dv = torch.zeros(2 * 30000 * 64, dtype=torch.bfloat16, device=DEV)
    job.dmask = None
    job.ws = job.ws[:16]
    with pytest.raises(ckv.ChunkKVError) as e:
        job.call()
    assert e.value.status == 4
