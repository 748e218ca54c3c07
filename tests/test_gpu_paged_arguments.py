"""Arguments that are not there: refused by the calls over pages as by the others, and not asked for where they are not needed."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests import paged_helpers as H

pytestmark = pytest.mark.gpu
DEV = H.DEV
NULL = 1


def state():
    gen = torch.Generator().manual_seed(1)
    cache = H.Cache(gen, ckv.BF16, 4, 2, 64, 16, [40], [10])
    qkv = torch.randn((3, 8, 64), generator=gen).bfloat16().to(DEV)
    return cache, dict(table=cache.table.to(DEV), kp=cache.pool(cache.k), vp=cache.pool(cache.v), n=cache.len.to(DEV), pos=cache.pos.to(DEV), w=cache.weight.to(DEV), qkv=qkv,
                       at=torch.arange(3, dtype=torch.int32, device=DEV), q_out=torch.zeros((3, 4, 64), dtype=torch.bfloat16, device=DEV))


def refused(call, **missing):
    with pytest.raises(ckv.ChunkKVError) as e:
        call(**missing)
    assert e.value.status == NULL


def test_append(lib):
    cache, s = state()
    good = dict(q=s["qkv"][:, :4], k=s["qkv"][:, 4:6], v=s["qkv"][:, 6:], at=s["at"], q_out=s["q_out"], table=s["table"], kp=s["kp"][0], vp=s["vp"][0], n=s["n"][0], after=s["n"][0])

    def call(new=(3,), **kw):
        x = {**good, **kw}
        ckv.chunkkv_paged_append(cache.pages, new, x["q"], x["k"], x["v"], x["at"], None, None, 0.0, None, False, x["q_out"], x["table"], x["kp"], x["vp"], x["n"], x["after"], None, None)

    for name in good:
        refused(call, **{name: None})
    before = s["n"].clone()
    call((0,), q=None, k=None, v=None, at=None, q_out=None)   # a step without tokens needs no arrays of them
    assert torch.equal(s["n"], before)
    call()
    assert torch.equal(s["n"], before + 3)


def test_attention(lib):
    cache, s = state()
    ws = torch.empty(ckv.chunkkv_paged_decode_workspace_bytes(cache.pages, False), dtype=torch.uint8, device=DEV)
    good = dict(table=s["table"], q=s["q_out"][:1], kp=s["kp"][0], vp=s["vp"][0], out=torch.zeros((1, 4, 64), device=DEV))

    def call(**kw):
        x = {**good, **kw}
        ckv.chunkkv_paged_decode_attention(cache.pages, x["table"], None, x["q"], x["kp"], x["vp"], x["out"], None, None, ws)

    for name in good:
        refused(call, **{name: None})


@pytest.mark.parametrize("layers", [1, 6])
def test_stacks(lib, layers):
    """A pool or a cache that is not there, first or last in lists short and long; lists that are not there."""
    gen = torch.Generator().manual_seed(2)
    cache = H.Cache(gen, ckv.BF16, 2, 1, 64, 16, [80], [0], layers=layers)
    prob = ckv.Problem(2, 1, 64, 16, 8, ckv.BF16, [200], [64], [0], 200 * 64, 64)
    full = [torch.zeros(200 * 64, dtype=torch.bfloat16, device=DEV) for _ in range(layers)]
    sel = [torch.zeros((layers, prob.sel_cap), dtype=torch.int32, device=DEV) for _ in range(2)] + [torch.zeros(layers, dtype=torch.int32, device=DEV)]
    up = dict(table=cache.table.to(DEV), kp=cache.pool(cache.k), vp=cache.pool(cache.v), n=cache.len.to(DEV), pos=cache.pos.to(DEV), w=cache.weight.to(DEV))
    imp = [torch.zeros(prob.score_cap * 8, device=DEV) for _ in range(layers)]
    good = dict(up, k=full, v=full, chunks=sel[0], lens=sel[1], count=sel[2], imp=imp)
    ws = torch.empty(ckv.chunkkv_paged_evict_workspace_bytes(cache.pages, layers, [70]), dtype=torch.uint8, device=DEV)

    def compact(**kw):
        x = {**good, **kw}
        ckv.chunkkv_paged_compact(prob, cache.pages, 1, x["k"], x["v"], x["chunks"], x["lens"], x["count"], x["imp"], x["table"], x["kp"], x["vp"], x["n"], None, None)

    def evict(**kw):
        x = {**good, **kw}
        ckv.chunkkv_paged_evict(cache.pages, [70], 3, x["table"], x["kp"], x["vp"], x["n"], x["pos"], x["w"], ws)

    for name in ("chunks", "lens", "count", "table", "n"):
        refused(compact, **{name: None})
    for name in ("table", "n", "pos", "w"):
        refused(evict, **{name: None})
    for at in (0, layers - 1):
        for name, call in (("k", compact), ("v", compact), ("kp", compact), ("vp", compact), ("imp", compact), ("kp", evict), ("vp", evict)):
            ts = list(good[name])
            ts[at] = None
            refused(call, **{name: ts})
    compact()
    evict()
