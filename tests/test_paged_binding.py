"""Checks of the binding of the calls over pages that need no GPU."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from paper_2502_00299_amd import binding

ROOM = 4 * 2 * 16 * 64


def pools(layers, kind=torch.bfloat16):
    return [torch.zeros(4, 2, 16, 64, dtype=kind) for _ in range(layers)]


@pytest.mark.parametrize("layers", [1, 4, 5, 32])
@pytest.mark.parametrize("kind", [torch.float16, torch.float32, torch.int16])
@pytest.mark.parametrize("place", [0, -1])
def test_every_pool_of_a_stack_has_the_type(layers, kind, place):
    """A pool of another type is refused wherever it is in the list, also where it has as many bytes or more."""
    ts = pools(layers)
    assert list(binding._pools("here", -1, "k_pages", ts, torch.bfloat16, ROOM)) == [t.data_ptr() for t in ts]
    ts[place] = torch.zeros(4, 2, 16, 64, dtype=kind)
    with pytest.raises(ValueError, match="k_pages is torch"):
        binding._pools("here", -1, "k_pages", ts, torch.bfloat16, ROOM)


@pytest.mark.parametrize("layers", [1, 2, 3, 32])
@pytest.mark.parametrize("kind", [torch.float16, torch.float32])
def test_two_lists_of_pools(layers, kind):
    ks, vs = pools(layers), pools(layers)
    at, k, v = binding._pool_pairs("here", -1, ("k_pages", "v_pages"), ks, vs, torch.bfloat16, ROOM)
    assert list(at) == [t.data_ptr() for t in ks + vs] and (k, v) == (at.buffer_info()[0], at.buffer_info()[0] + 8 * layers)
    for name, ts in (("k_pages", ks), ("v_pages", vs)):
        for wrong, why in ((torch.zeros(4, 2, 16, 64, dtype=kind), "is torch"), (torch.zeros(3, 2, 16, 64, dtype=torch.bfloat16), "has")):
            good, ts[-1] = ts[-1], wrong
            with pytest.raises(ValueError, match=f"{name} {why}"):
                binding._pool_pairs("here", -1, ("k_pages", "v_pages"), ks, vs, torch.bfloat16, ROOM)
            ts[-1] = good
    with pytest.raises(ValueError, match="k_pages is on device"):
        binding._pool_pairs("here", 0, ("k_pages", "v_pages"), ks, vs, torch.bfloat16, ROOM)


def test_problems_without_sequences_are_the_library_s_to_refuse():
    p = ckv.Problem(4, 2, 64, 16, 8, ckv.BF16, [], [], [], 64, 64, out_base=[], sel_cap=1, score_cap=1)
    assert ckv.chunkkv_workspace_bytes(p, 1, 1) == 0 and ckv.chunkkv_decode_workspace_bytes(p, False) == 0


def test_reach_of_full_caches():
    """What has to be behind a cache's first element: by every sequence that the library sees, one past a short list of bases too."""
    d, hkv = 64, 2
    prob = ckv.Problem(4, hkv, d, 16, 8, ckv.BF16, [100, 40], [8, 8], [0, 100 * hkv * d], d, hkv * d)
    prob._c()
    assert prob._kept[3] == 140 * hkv * d
    prob.seqlen, prob.kv_base = [100, 4000], [0]
    prob._c()
    assert prob._kept[1].kv_base[1] == 0 and prob._kept[3] == 4000 * hkv * d


GOOD = dict(n_q_heads=32, n_kv_heads=8, head_dim=128, dtype=ckv.BF16, page_tokens=16, n_pages=100, max_tokens=[848, 17])


@pytest.mark.parametrize("name", ["n_q_heads", "n_kv_heads", "page_tokens", "n_pages", "table_pitch", "slot_pitch", "max_tokens"])
@pytest.mark.parametrize("off", [1 << 32, -(1 << 32)])
def test_numbers_that_do_not_fit(name, off):
    """Sizes of which the library would see the lower 32 bits alone, fewer than none for the checks."""
    p = ckv.Pages(**GOOD)
    assert ckv.chunkkv_paged_decode_workspace_bytes(p, True) > 0
    setattr(p, name, [848, 17 + off] if name == "max_tokens" else getattr(p, name) + off)
    with pytest.raises(ValueError, match="does not fit"):
        ckv.chunkkv_paged_decode_workspace_bytes(p, True)


def test_strides_that_do_not_fit():
    with pytest.raises(ValueError, match="does not fit"):
        ckv.chunkkv_paged_decode_workspace_bytes(ckv.Pages(**GOOD, stride_tok=128, stride_head=2048, stride_page=(1 << 64) + 16384), True)


def test_host_numbers_that_do_not_fit():
    for numbers in ([(1 << 32) + 3, 1], [1 - (1 << 32), 2]):
        with pytest.raises(ValueError, match="does not fit"):
            binding._ints(numbers)
    assert list(binding._ints([3, 2 ** 31 - 1])[1]) == [3, 2 ** 31 - 1]


@pytest.mark.parametrize("tokens", [0, 1])
@pytest.mark.parametrize("pitch", [0, 1, 385, 4096])
def test_rows_without_a_next_one(tokens, pitch):
    """The stride of an axis of one token is not looked at: rows of 384 elements, 385 apart in something longer."""
    x = torch.zeros(9000, dtype=torch.bfloat16).as_strided((tokens, 3, 128), (pitch, 128, 1))
    at, stride = binding._new_rows("here", -1, "k", x, torch.bfloat16, tokens, 3, 128)
    assert stride == 384 and at == x.data_ptr()
    y = torch.zeros(9000, dtype=torch.bfloat16).as_strided((2, 3, 128), (400, 128, 1))
    assert binding._new_rows("here", -1, "k", y, torch.bfloat16, 2, 3, 128) == (y.data_ptr(), 400)
