"""Softmax weights of 16-bit types where a segment has up to 32 query rows: outputs are off by their own rounding and what fp32 is, so elements near zero
beside large values are right too; nothing of the size of a rounded weight is left in them."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests.rows_helpers import HALF_STEP, attend, near, near_lse
from tests.test_gpu_cross import Job as CrossJob
from tests.test_gpu_cross import random_mask
from tests.test_gpu_shared import Job as SharedJob

pytestmark = pytest.mark.gpu
TYPES = [ckv.BF16, ckv.F16]


def fine(q, k, v, scale, dtype):
    """As attend(), with weights of two numbers: the second takes in what the first leaves, to half a step of that (2^-16 of the weight in bf16, 2^-22 in fp16;
    or half the smallest fp16, 2^-25 beside a reference of 2^9, which is 2^-34 of the largest weight at most), and an output is a mean of values.  Its own
    rounding: half a step, or half the smallest fp16."""
    out, lse, bound, lbound = attend(q, k, v, scale, ckv.F32)
    if len(k):
        u, top = HALF_STEP[dtype], v.abs().max()
        bound = bound + u * u * top
        if dtype == ckv.F16:
            x = q @ k.t() * scale
            bound = bound + len(k) * 2.0 ** -34 * torch.exp(x.amax(1) - lse)[:, None] * top
        bound = bound + u * (out.abs() + bound) + (2.0 ** -25 if dtype == ckv.F16 else 0.0)
    return out, lse, bound, lbound


def small_outputs(rows):
    """Half of the values of every head with either sign, so that outputs are small beside them."""
    for k, v in rows:
        v[1::2] = -v[:-1:2] if len(v) % 2 == 0 else -v[:-2:2]


def check(job, out, lse, bound, lbound):
    job.device().call()
    torch.cuda.synchronize()
    result = job.result() if hasattr(job, "result") else job.out
    near(result, out, bound, "out")
    near_lse(job.lse[:len(lse)], lse, lbound, "lse")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("states,masked", [(2, False), (33, False), (150, True), (700, False), (5000, False), (9001, True)])
def test_cross(lib, dtype, d, states, masked):
    for hq, hkv, tokens in ((8, 2, [1, 8, 0, 5]), (3, 3, [32, 1]), (32, 1, [1])):
        job = CrossJob(states, dtype, hq, hkv, d, tokens, [states] * len(tokens), layout="heads", mask=random_mask(0.3) if masked else None)
        g = hq // hkv
        parts = [torch.zeros((job.T, hq, d), dtype=torch.float64), torch.zeros((job.T, hq), dtype=torch.float64), torch.zeros((job.T, hq, d), dtype=torch.float64),
                 torch.zeros((job.T, hq), dtype=torch.float64)]
        t = 0
        for b, n in enumerate(tokens):
            for h in range(hkv if n else 0):
                k, v = job.rows[b, h]
                small_outputs([(k, v)])
                at = torch.arange(states)
                if masked:
                    at = at[job.mask[b, :states] != 0]
                at = (job.base[b] + h * job.sh + at * job.st)[:, None] + torch.arange(d)
                job.v[at.flatten()] = v.to(job.v.dtype).flatten()
                got = fine(job.q[t:t + n, h * g:(h + 1) * g].double().flatten(0, 1), k, v, d ** -0.5, dtype)
                for to, x in zip(parts, got):
                    to[t:t + n, h * g:(h + 1) * g] = x.view(n, g, *x.shape[1:])
            t += n
        check(job, *parts)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("prefix,sharing,own", [([40, 700], [3, 5], [1, 0, 70, 16, 5, 300, 2, 33]), ([3000], [8], [20] * 8), ([1, 0], [1, 2], [0, 1, 900])])
def test_behind_prefixes(lib, dtype, d, prefix, sharing, own):
    job = SharedJob(3, dtype, 8, 2, d, 16, prefix, sharing, own)
    parts = [torch.zeros((job.B, 8, d), dtype=torch.float64), torch.zeros((job.B, 8), dtype=torch.float64), torch.zeros((job.B, 8, d), dtype=torch.float64), torch.zeros((job.B, 8), dtype=torch.float64)]
    for i, heads in enumerate(job.rows):
        for h, (k, v) in enumerate(heads):
            small_outputs([(k, v)])
            s = torch.arange(len(v))
            job.v[(job.prefix_table[i] if i < job.P else job.table[i - job.P]).long()[s // 16], h, s % 16] = v.to(job.v.dtype)
    b = 0
    for i, n in enumerate(sharing):
        for b in range(b, b + n):
            for h in range(2):
                k, v = (torch.cat(x) for x in zip(job.rows[i][h], job.rows[job.P + b][h]))
                for to, x in zip(parts, fine(job.q[b, 4 * h:4 * h + 4].double(), k, v, d ** -0.5, dtype)):
                    to[b, 4 * h:4 * h + 4] = x
        b += n > 0
    check(job, *parts)
