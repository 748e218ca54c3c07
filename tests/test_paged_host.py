"""Calls over caches in pages, without a GPU: argument checks, workspace sizes, the kept struct, the oracle's own pins."""
import copy
import ctypes as C
import os
import pickle
import subprocess

import numpy as np
import pytest
import torch

import paper_2502_00299_amd as ckv
from oracle import paged_oracle as orc

FAKE = C.c_void_p(0x1000)   # never dereferenced: every call below fails a check before a launch
ODD = C.c_void_p(0x1008)
OK, NULL, SHAPE, UNSUPPORTED, WORKSPACE = range(5)


@pytest.fixture(scope="module")
def lib():
    return ckv.load_library()


def good(**kw):
    d = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=ckv.BF16, page_tokens=16, n_pages=100, max_tokens=[848, 17])
    d.update(kw)
    return ckv.Pages(**d)


def attend(lib, p, table=FAKE, q=FAKE, k=FAKE, v=FAKE, out=FAKE, weight=None, ws=FAKE, size=1 << 40):
    return lib.chunkkv_paged_decode_attention(C.byref(p.as_c()), table, None, q, k, v, out, None, weight, ws, size, None)


def append(lib, p, new=(1, 1), q=FAKE, q_tok=4096, k=FAKE, k_tok=1024, v=FAKE, v_tok=1024, positions=FAKE, q_norm=None, k_norm=None, eps=0.0, freq=FAKE,
           rotary=128, q_out=FAKE, table=FAKE, kp=FAKE, vp=FAKE, n=FAKE, n_out=FAKE):
    new = None if new is None else (C.c_int32 * len(new))(*new)
    return lib.chunkkv_paged_append(C.byref(p.as_c()), new, q, q_tok, k, k_tok, v, v_tok, positions, q_norm, k_norm, eps, freq, rotary, 0, q_out, table, kp, vp,
                                    n, n_out, None, None, None)


def evict(lib, p, layers=2, budget=(800, 16), recent=4, table=FAKE, k=FAKE, v=FAKE, n=FAKE, pos=FAKE, weight=FAKE, ws=FAKE, size=1 << 40):
    ks, vs = ((C.c_void_p * layers)(*[x] * layers) if layers > 0 else None for x in (k, v))
    budget = None if budget is None else (C.c_int32 * len(budget))(*budget)
    return lib.chunkkv_paged_evict(C.byref(p.as_c()), layers, budget, recent, table, ks, vs, n, pos, weight, ws, size, None)


@pytest.mark.parametrize("kw,status", [
    (dict(n_q_heads=30), SHAPE), (dict(n_kv_heads=0), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_tokens=[-1, 3]), SHAPE), (dict(softmax_scale=-1.0), SHAPE),
    (dict(softmax_scale=float("nan")), SHAPE), (dict(softmax_scale=float("inf")), SHAPE), (dict(table_pitch=52), SHAPE), (dict(slot_pitch=847), SHAPE),
    (dict(stride_tok=64), SHAPE), (dict(stride_tok=132), SHAPE), (dict(stride_tok=128, stride_head=2052, stride_page=16384), SHAPE),
    (dict(stride_tok=128, stride_head=2048, stride_page=-8), SHAPE),
    (dict(head_dim=96), UNSUPPORTED), (dict(dtype=3), UNSUPPORTED), (dict(page_tokens=8), UNSUPPORTED), (dict(page_tokens=24), UNSUPPORTED),
    (dict(page_tokens=4112), UNSUPPORTED), (dict(n_q_heads=257, n_kv_heads=1), UNSUPPORTED), (dict(max_tokens=[(1 << 24) + 1]), UNSUPPORTED),
    (dict(stride_tok=1 << 22, stride_head=128, stride_page=1 << 26), UNSUPPORTED), (dict(n_q_heads=4096, n_kv_heads=4096), UNSUPPORTED),
])
def test_pages_that_are_refused(lib, kw, status):
    p = good(**kw)
    assert ckv.chunkkv_paged_decode_workspace_bytes(p, True) == 0
    assert ckv.chunkkv_paged_evict_workspace_bytes(p, 1, [0] * p.batch) == 0
    assert attend(lib, p) == status
    assert append(lib, p, [1] * p.batch, q_tok=1 << 20, k_tok=1 << 20, v_tok=1 << 20, rotary=32) == status
    assert evict(lib, p, budget=[0] * p.batch, recent=0) == status


def test_null_pages(lib):
    assert lib.chunkkv_paged_decode_workspace_bytes(None, 0) == 0
    assert lib.chunkkv_paged_decode_attention(None, FAKE, None, FAKE, FAKE, FAKE, FAKE, None, None, FAKE, 1 << 40, None) == NULL
    cp = good().as_c()
    cp.max_tokens = C.POINTER(C.c_int32)()
    assert lib.chunkkv_paged_decode_workspace_bytes(C.byref(cp), 0) == 0


def test_attention_arguments(lib):
    p = good()
    for name in ("table", "q", "k", "v", "out"):
        assert attend(lib, p, **{name: None}) == NULL
    for name in ("q", "k", "v"):
        assert attend(lib, p, **{name: ODD}) == SHAPE
    need, more = ckv.chunkkv_paged_decode_workspace_bytes(p, False), ckv.chunkkv_paged_decode_workspace_bytes(p, True)
    assert 0 < need < more
    assert attend(lib, p, ws=None) == WORKSPACE and attend(lib, p, size=need - 1) == WORKSPACE and attend(lib, p, weight=FAKE, size=more - 1) == WORKSPACE
    assert attend(lib, p, ws=C.c_void_p(0x1004)) == WORKSPACE


def test_workspace_of_a_long_batch(lib):
    """Scores of every slot and head, partial results of every range: nothing grows with the longest sequence times the batch."""
    p = good(max_tokens=[1 << 20] + [100] * 200, n_pages=70000)
    assert ckv.chunkkv_paged_decode_workspace_bytes(p, True) < (1 << 20) * 32 * 4 * 1.3 + (64 << 20)


def test_append_arguments(lib):
    p = good()
    for name in ("new", "k", "v", "positions", "table", "kp", "vp", "n", "n_out"):
        assert append(lib, p, **{name: None}) == NULL
    assert append(lib, p, q=None) == NULL and append(lib, p, q_out=None) == NULL and append(lib, p, freq=None) == NULL
    assert append(lib, p, q=None, q_out=None, q_norm=FAKE) == NULL
    for name in ("q", "k", "v", "q_norm", "k_norm", "q_out", "kp", "vp"):
        assert append(lib, p, **{name: ODD}) == SHAPE
    assert append(lib, p, new=(1, -1)) == SHAPE
    assert append(lib, p, q_tok=4088) == SHAPE and append(lib, p, k_tok=1016) == SHAPE and append(lib, p, v_tok=1028) == SHAPE
    assert append(lib, p, rotary=-16) == SHAPE and append(lib, p, rotary=144) == SHAPE and append(lib, p, rotary=0) == SHAPE
    assert append(lib, p, rotary=24) == UNSUPPORTED
    assert append(lib, p, eps=-1.0) == SHAPE and append(lib, p, eps=float("nan")) == SHAPE
    assert append(lib, p, new=(1 << 24, 1)) == UNSUPPORTED


def test_evict_arguments(lib):
    p = good()
    for name in ("budget", "table", "n", "pos", "weight", "k", "v"):
        assert evict(lib, p, **{name: None}) == NULL
    assert evict(lib, p, k=ODD) == SHAPE and evict(lib, p, v=ODD) == SHAPE
    assert evict(lib, p, layers=0) == SHAPE and evict(lib, p, recent=-1) == SHAPE and evict(lib, p, recent=17) == SHAPE and evict(lib, p, budget=(5, -1), recent=0) == SHAPE
    need = ckv.chunkkv_paged_evict_workspace_bytes(p, 2, [800, 16])
    assert need >= 2 * 2 * 8 * (2 * 48) * 4          # 48 slots of the longer sequence can move
    assert evict(lib, p, ws=None) == WORKSPACE and evict(lib, p, size=need - 1) == WORKSPACE


def test_compact_arguments(lib):
    p = good(max_tokens=[848])
    prob = ckv.Problem(32, 8, 128, 32, 10, ckv.BF16, [8192], [816], [0], 8192 * 128, 128)

    def call(prob=prob, p=p, n=2, reuse=1, k=FAKE, kp=FAKE, sel=FAKE, imp=None, table=FAKE, length=FAKE):
        tab = [(C.c_void_p * 2)(x, x) for x in (k, FAKE, kp, FAKE)]
        return lib.chunkkv_paged_compact(C.byref(prob.as_c()), C.byref(p.as_c()), n, reuse, tab[0], tab[1], sel, FAKE, FAKE, imp, table, tab[2], tab[3],
                                         length, None, None, None)

    assert call(k=None) == NULL and call(kp=None) == NULL and call(sel=None) == NULL and call(table=None) == NULL and call(length=None) == NULL
    assert call(imp=(C.c_void_p * 2)(0x1000, None)) == NULL
    assert call(k=ODD) == SHAPE and call(kp=ODD) == SHAPE and call(n=0) == SHAPE and call(reuse=0) == SHAPE
    assert call(p=good(max_tokens=[847])) == SHAPE                  # 816 + 32 rows
    assert call(p=good(max_tokens=[848, 848])) == SHAPE and call(p=good(max_tokens=[848], dtype=ckv.F16)) == SHAPE
    assert call(p=good(max_tokens=[848], head_dim=64)) == SHAPE and call(p=good(max_tokens=[848], n_q_heads=16)) == SHAPE
    assert call(prob=ckv.Problem(32, 8, 128, 32, 10, ckv.BF16, [16], [0], [0], 8192 * 128, 128)) == SHAPE


def test_kept_struct_follows_changes(lib):
    p = good()
    a = ckv.chunkkv_paged_decode_workspace_bytes(p, True)
    p.max_tokens[1] = 900
    p.slot_pitch = 900
    p.table_pitch = 60
    assert ckv.chunkkv_paged_decode_workspace_bytes(p, True) > a
    assert ckv.Pages(**vars(p)) == p
    for q in (copy.deepcopy(p), pickle.loads(pickle.dumps(p))):
        assert q == p
        q.max_tokens[0] = 1
        assert p._c()._obj.max_tokens[0] == 848 and q._c()._obj.max_tokens[0] == 1
    with pytest.raises(ValueError):
        ckv.chunkkv_paged_evict_workspace_bytes(p, 1, [5])


def test_oracle_rotation_and_norm():
    """Rotation keeps the length of every pair; a position difference is what a product of rotated rows depends on; a
    constant row has norm 1."""
    rng = np.random.default_rng(1)
    freq = 10000.0 ** (-np.arange(16) / 16)
    x, y = rng.standard_normal(64), rng.standard_normal(64)
    for inter in (False, True):
        turn = lambda z, p: orc.norm_and_rotate(z, None, 0.0, p, freq, inter)  # noqa: E731
        assert np.allclose(turn(x, 0), x) and np.allclose(np.linalg.norm(turn(x, 77)), np.linalg.norm(x)) and np.array_equal(turn(x, 5)[32:], x[32:])
        assert np.isclose(turn(x, 900) @ turn(y, 880), turn(x, 20) @ turn(y, 0))
    assert np.allclose(orc.norm_and_rotate(np.full(64, 3.0), np.arange(64.0), 0.0, 0, None, False), np.arange(64.0))


def test_oracle_attention_and_eviction():
    torch.manual_seed(2)
    q, k, v = torch.randn(3, 64, dtype=torch.float64), torch.randn(20, 64, dtype=torch.float64), torch.randn(20, 64, dtype=torch.float64)
    out, lse, p = orc.attention(q.numpy(), k.numpy(), v.numpy(), 0.125)
    want = torch.nn.functional.scaled_dot_product_attention(q[None], k[None], v[None], scale=0.125)[0]
    assert np.allclose(out, want.numpy()) and np.allclose(p.sum(1), 1) and np.allclose(lse, torch.logsumexp(0.125 * q @ k.t(), 1).numpy())
    weight, pos = [5.0, 1.0, 4.0, 1.0, 9.0, 0.0], [0, 1, 2, 3, 4, 5]
    assert orc.evict(weight, pos, 6, 6, 0) == (6, [])
    assert orc.evict(weight, pos, 6, 3, 0) == (3, [(4, 1)])             # 9, 5, 4
    assert orc.evict(weight, pos, 6, 3, 1) == (3, [(4, 1), (5, 2)])     # the newest in any case
    assert orc.evict([1.0] * 6, pos, 6, 2, 0) == (2, [])                # ties: the lower slots
    assert orc.evict(weight, pos, 6, 0, 0) == (0, [])


@pytest.mark.parametrize("layers", [3, 6])
def test_pools_of_a_stack_are_measured(layers):
    from paper_2502_00299_amd import binding
    pools = [torch.zeros(4, 2, 16, 64, dtype=torch.bfloat16) for _ in range(layers)]
    at = binding._pools("here", -1, "k_pages", pools, torch.bfloat16, 4 * 2 * 16 * 64)
    assert list(at) == [t.data_ptr() for t in pools]
    bigger = torch.zeros(9, 4, 16, 64, dtype=torch.bfloat16)
    views = pools[:-1] + [bigger[1:5, :2]]   # not contiguous, but with as much memory behind it
    assert binding._pools("here", -1, "k_pages", views, torch.bfloat16, 4 * 2 * 16 * 64)[-1] == bigger[1].data_ptr()
    for wrong in (torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16).expand(4, 2, 16, 64)):
        with pytest.raises(ValueError, match="k_pages has"):
            binding._pools("here", -1, "k_pages", pools[:-1] + [wrong], torch.bfloat16, 4 * 2 * 16 * 64)
    with pytest.raises(ValueError, match="on device"):
        binding._pools("here", 0, "k_pages", pools, torch.bfloat16, 16)


def test_checks_and_plans_are_clean_under_asan_and_ubsan(tmp_path):
    from paper_2502_00299_amd import build
    exe = build.build_host_sanitizer_check(str(tmp_path), "host_sanitizer_pages")
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=0", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300, env=env)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "HOST SANITIZER RUN OK" in r.stdout, out[-4000:]
    assert "AddressSanitizer" not in out and "runtime error" not in out, out[-4000:]
