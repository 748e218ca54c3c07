"""Attention of many query rows over the same keys in 64 bits, and how far the library's may be from it."""
import math

import torch

import paper_2502_00299_amd as ckv

DEV = "cuda:0"
KIND = {ckv.F32: torch.float32, ckv.BF16: torch.bfloat16, ckv.F16: torch.float16}
HALF_STEP = {ckv.F32: 2.0 ** -24, ckv.BF16: 2.0 ** -8, ckv.F16: 2.0 ** -11}


def attend(q, k, v, scale, dtype):
    """Rows q [n][d] over keys k, v [m][d], all float64 -> output, log-sum-exp, and the bound of either's error.

    Scores: d products and as many sums in fp32, so off by (d + 4) 2^-24 of sum |q_i k_i| at most, and the argument of the exponential by
    two roundings (2^-23) of the largest difference of scores, in natural units.  A weight is off by that, relatively; a sum of n weights by
    n / 16 + 40 roundings (16 of a lane in two or four chains, tile after tile, ranges and halves).  An output is a mean of values, so an error e of
    all weights (and of their sum) moves it by 2 e of the largest value.  Weights of 16 bits add their rounding u (fp16 2^-33 of the largest
    weight each beside it), the output its own."""
    n, d = k.shape
    u = HALF_STEP[dtype]
    if n == 0:
        zero = torch.zeros(q.shape[0], dtype=torch.float64)
        return torch.zeros_like(q), zero - math.inf, torch.zeros_like(q), zero
    x = q @ k.t() * scale
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    out = p @ v
    size = (q.abs() @ k.abs().t()).amax(1) * scale
    delta = (d + 4) * 2.0 ** -24 * size + 2.0 ** -23 * (x.amax(1) - x.amin(1)).clamp(max=90.0) + 2.0 ** -23 * x.abs().amax(1)
    sums = (n / 16 + 40) * 2.0 ** -24
    e = 2 * (torch.expm1(delta) + sums)
    top = v.abs().max()
    small = 0.0
    if dtype != ckv.F32:
        e = e + 2 * u
        small = u * out.abs()
    if dtype == ckv.F16:
        e = e + n * 2.0 ** -33 * torch.exp(x.amax(1) - lse)
        small = small + 2.0 ** -25
    return out, lse, e[:, None] * top + small + 2.0 ** -23 * top, delta + sums + 2.0 ** -22 * lse.abs() + 2.0 ** -22


def near(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    bad = ~(err <= bound)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound, first at {bad.nonzero()[0].tolist()}, error {err[bad][0]}, bound {bound.expand_as(err)[bad][0]}"


def near_lse(got, want, bound, what):
    got = got.double().cpu()
    none = want == -math.inf
    assert (got[none] == -math.inf).all(), f"{what}: rows without a key"
    near(got[~none], want[~none], bound[~none], what)
