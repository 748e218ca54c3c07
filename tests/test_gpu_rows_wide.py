"""Attention of many rows in the forms that small calls do not take (tests/rows_shapes.py): workgroups of 256 query rows over many tiles and ranges,
under masks, over pages; more segments than a launch has, each launch with ranges that are joined.  Against float64, formed on the device."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import rows_shapes as shapes
from tests.rows_helpers import DEV, attend
from tests.test_gpu_cross import Job as CrossJob
from tests.test_gpu_cross import edges_mask, random_mask
from tests.test_gpu_shared import Job as SharedJob

pytestmark = pytest.mark.gpu
TYPES = [ckv.BF16, ckv.F16, ckv.F32]


def on_device(q, k, v, scale, dtype):
    return [x.cpu() for x in attend(q.to(DEV).double(), k.to(DEV), v.to(DEV), scale, dtype)]


class Cross(CrossJob):
    def want(self):
        g, s = self.hq // self.hkv, self.scale or self.d ** -0.5
        out, bound = (torch.zeros((self.T, self.hq, self.d), dtype=torch.float64) for _ in range(2))
        lse, lbound = (torch.zeros((self.T, self.hq), dtype=torch.float64) for _ in range(2))
        t = 0
        for b, n in enumerate(self.q_len):
            for h in range(self.hkv if n else 0):
                heads = slice(h * g, (h + 1) * g)
                got = on_device(self.q[t:t + n, heads].flatten(0, 1), *self.rows[b, h], s, self.dtype)
                for to, x in zip((out, lse, bound, lbound), got):
                    to[t:t + n, heads] = x.view(n, g, *x.shape[1:])
            t += n
        return out, lse, bound, lbound


class Shared(SharedJob):
    def want(self):
        g, s = self.hq // self.hkv, self.scale or self.d ** -0.5
        out, bound = (torch.zeros((self.B, self.hq, self.d), dtype=torch.float64, device=DEV) for _ in range(2))
        lse, lbound = (torch.zeros((self.B, self.hq), dtype=torch.float64, device=DEV) for _ in range(2))
        q, first = self.q.to(DEV).double(), 0
        for i, n in enumerate(self.sharing):
            for h in range(self.hkv if n else 0):
                heads, whole = slice(h * g, (h + 1) * g), [x.to(DEV) for x in self.rows[i][h]]
                for b in range(first, first + n):
                    k, v = (torch.cat((x, y.to(DEV))) for x, y in zip(whole, self.rows[self.P + b][h]))
                    for to, x in zip((out, lse, bound, lbound), attend(q[b, heads], k, v, s, self.dtype)):
                        to[b, heads] = x.to(DEV)
            first += n
        return [x.cpu() for x in (out, lse, bound, lbound)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [None, random_mask(0.1), random_mask(0.97)], ids=["whole", "holes", "few"])
def test_256_rows(lib, dtype, d, mask):
    """More tiles than the ring has, in one range: the last workgroup's rows end inside a wavefront."""
    hq, hkv, n, m, _, _ = shapes.WIDE_CROSS[0]
    Cross(1, dtype, hq, hkv, d, [n], [m], layout="padded", mask=mask).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", shapes.WIDE_CROSS[1:], ids=["ranges", "whole"])
@pytest.mark.parametrize("masked", [False, True])
def test_256_rows_and_windows(lib, dtype, d, shape, masked):
    """More blocks than a window of places; wavefronts without rows; partial rows.  Heads of other lengths, one of them none, beside a mask."""
    hq, hkv, n, m, _, _ = shape
    lens = [[(h * 977) % (m + 1) if h % 3 else m for h in range(hkv)]] if masked else None
    Cross(2, dtype, hq, hkv, d, [n], [m], layout="heads", mask=random_mask(0.3) if masked else None, lens=lens).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_256_rows_beside_few(lib, dtype, d):
    """Sequences of unlike lengths, without states or queries, and of a few rows: their workgroups are split in two."""
    hq, hkv, q_len, states = shapes.WIDE_RAGGED
    Cross(3, dtype, hq, hkv, d, q_len, states, layout="packed").check()


@pytest.mark.parametrize("dtype", TYPES)
def test_256_rows_under_the_edges_of_a_mask(lib, dtype):
    """No state; the first; the last; one tile in the middle; one of every tile."""
    hq, hkv, n, m, _, _ = shapes.WIDE_CROSS[0]
    Cross(4, dtype, hq, hkv, 128, [n] * 5, [m] * 5, layout="padded", mask=edges_mask).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("shape", shapes.WIDE_SHARED, ids=["ring", "groups", "windows"])
def test_256_rows_of_a_prefix(lib, dtype, d, shape):
    """Pages of 48 slots, three blocks: they end inside tiles.  Heads of unlike lengths; pages that are not there."""
    hq, hkv, n, m, _ = shape
    Shared(5, dtype, hq, hkv, d, 48, [m], [n], shapes.own_slots(n), uneven=True, missing=[(0, 1), (0, 30), (0, m // 48), (3, 0)]).check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_launches_with_ranges(lib, dtype, d):
    """Every launch of a cross attention has partial rows in the same workspace: joined before the next launch writes its own.  Lengths and masks that differ
    from sequence to sequence, lse behind those of the launches before."""
    q_len, states = shapes.many_sequences()
    job = Cross(6, dtype, 4, 2, d, q_len, states, layout="packed")
    assert ckv.chunkkv_cross_workspace_bytes(job.plan) > 256
    job.check()
    lens = [[max(0, n - 7 * b % 50), n - 3 * b % 40] for b, n in enumerate(states)]
    job = Cross(7, dtype, 4, 2, d, q_len, states, layout="heads", lens=lens, mask=random_mask(0.2))
    assert ckv.chunkkv_cross_workspace_bytes(job.plan) > 256
    job.check()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("d", [64, 128])
def test_launches_of_prefixes(lib, dtype, d):
    """Prefixes and sequences over several launches, long ones in each."""
    prefix, sharing, own = shapes.many_prefixes()
    Shared(8, dtype, 8, 2, d, 32, prefix, sharing, own, uneven=True).check()
