"""A document's cache from its projections to its readers: rotation, compression, pages, a question's tokens over the compressed cache,
and sequences that go on behind it token by token, eager and in a graph; every step against float64 on what the step was given."""
import pytest
import torch

import paper_2502_00299_amd as ckv
from tests.rows_helpers import DEV, KIND, attend, near, near_lse
from tests.test_gpu_rotate import check as check_rotation

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,d,captured", [(ckv.BF16, 128, True), (ckv.F16, 64, False), (ckv.F32, 64, True)])
def test_a_document_and_its_readers(lib, dtype, d, captured):
    kind, layers, L, w, c, hq, hkv, page, B, steps = KIND[dtype], 2, 1203, 16, 8, 8, 2, 16, 5, 4
    g, n_keep = hq // hkv, (L - w) // 5
    gen = torch.Generator(device=DEV).manual_seed(7)
    freq = ckv.chunkkv_rotary_frequencies(d, 500000.0, 4.0, 1.0, 32.0, 512.0).to(DEV)
    at = torch.arange(L, dtype=torch.int32, device=DEV)
    k, v, q_obs = [], [], []
    for _ in range(layers):
        qkv = torch.randn((L, hq + 2 * hkv, d), generator=gen, device=DEV).to(kind)
        cache, window = torch.zeros((hkv, L, d), dtype=kind, device=DEV), torch.zeros((1, hq, w, d), dtype=kind, device=DEV)
        ckv.chunkkv_rotate(None, qkv[:, hq:hq + hkv], at, freq, False, 1.1, None, cache.transpose(0, 1))
        ckv.chunkkv_rotate(qkv[L - w:, :hq], None, at[L - w:].clone(), freq, False, 1.1, window[0].transpose(0, 1), None)
        check_rotation(cache.transpose(0, 1)[None], qkv[None, :, hq:hq + hkv].cpu(), at[None].cpu(), freq.cpu(), False, 1.1, dtype)
        k.append(cache)
        v.append(qkv[:, hq + hkv:].transpose(0, 1).contiguous())
        q_obs.append(window)
    prob = ckv.Problem(hq, hkv, d, w, c, dtype, [L], [n_keep], [0], L * d, d)
    kept = n_keep + w
    k_out, v_out = ([torch.zeros((hkv, kept, d), dtype=kind, device=DEV) for _ in range(layers)] for _ in range(2))
    sel_chunk = torch.zeros((1, 1, hkv, prob.sel_cap), dtype=torch.int32, device=DEV)
    sel_len, sel_count = torch.zeros_like(sel_chunk), torch.zeros((1, 1, hkv), dtype=torch.int32, device=DEV)
    ws = torch.empty(ckv.chunkkv_workspace_bytes(prob, layers, 2), dtype=torch.uint8, device=DEV)
    ckv.chunkkv_compress_stack(prob, 2, [q_obs[0], None], k, v, k_out, v_out, sel_chunk, sel_len, sel_count, ws)

    # a question's tokens over the compressed cache
    q = torch.randn((7, hq, d), generator=gen, device=DEV).to(kind)
    plan = ckv.Cross(hq, hkv, d, dtype, [7], [kept], [0], prob.out_stride_head, prob.out_stride_tok)
    ws = torch.empty(ckv.chunkkv_cross_workspace_bytes(plan), dtype=torch.uint8, device=DEV)
    for layer in range(layers):
        out, lse = torch.zeros_like(q), torch.zeros((7, hq), device=DEV)
        ckv.chunkkv_cross_attention(plan, None, None, q, k_out[layer], v_out[layer], out, lse, ws)
        for h in range(hkv):
            heads = slice(h * g, (h + 1) * g)
            want = attend(q[:, heads].double().cpu().flatten(0, 1), k_out[layer][h].double().cpu(), v_out[layer][h].double().cpu(), d ** -0.5, dtype)
            near(out[:, heads].flatten(0, 1), want[0], want[2], "question")
            near_lse(lse[:, heads].flatten(), want[1], want[3], "question's lse")

    # the compressed cache as a prefix in pages, and sequences behind it
    room = steps + 1
    held, own = -(-kept // page), -(-room // page)
    n_pages = held + B * own + 1
    whole, pages = ckv.Pages(hq, hkv, d, dtype, page, n_pages, [kept]), ckv.Pages(hq, hkv, d, dtype, page, n_pages, [room] * B)
    order = torch.randperm(n_pages, generator=gen, device=DEV).int()
    prefix_table, table = order[:held][None].contiguous(), order[held:held + B * own].view(B, own).contiguous()
    kp, vp = ([torch.full((n_pages, hkv, page, d), float("nan"), dtype=kind, device=DEV) for _ in range(layers)] for _ in range(2))
    prefix_len, pos = torch.zeros((layers, 1, hkv), dtype=torch.int32, device=DEV), torch.zeros((layers, 1, hkv, whole.slot_pitch), dtype=torch.int32, device=DEV)
    ckv.chunkkv_paged_compact(prob, whole, 2, k, v, sel_chunk, sel_len, sel_count, None, prefix_table, kp, vp, prefix_len, pos, None)
    assert (prefix_len == kept).all()
    length = torch.zeros((layers, B, hkv), dtype=torch.int32, device=DEV)
    here = torch.full((B,), L, dtype=torch.int32, device=DEV)
    qkv = torch.randn((layers, B, hq + 2 * hkv, d), generator=gen, device=DEV).to(kind)
    q_rot, out = (torch.zeros((layers, B, hq, d), dtype=kind, device=DEV) for _ in range(2))
    lse = torch.zeros((layers, B, hq), device=DEV)
    ws = torch.empty(ckv.chunkkv_shared_decode_workspace_bytes(whole, pages, [B]), dtype=torch.uint8, device=DEV)

    def step():
        for i in range(layers):
            x = qkv[i]
            ckv.chunkkv_paged_append(pages, [1] * B, x[:, :hq], x[:, hq:hq + hkv], x[:, hq + hkv:], here, None, None, 0.0, freq, False, q_rot[i], table, kp[i], vp[i], length[i], length[i], None, None)
            ckv.chunkkv_shared_decode_attention(whole, pages, [B], prefix_table, prefix_len[i], table, length[i], q_rot[i], kp[i], vp[i], out[i], lse[i], ws)

    run = step
    if captured:
        step()               # one token, outside
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step()
        run = graph.replay
    for s in range(1 if captured else 0, steps):
        qkv.normal_(generator=gen)
        here.fill_(L + s)
        out.zero_()
        run()
        torch.cuda.synchronize()
        assert (length == s + 1).all()
        for i in range(layers):
            for b in range(B):
                for h in range(hkv):
                    heads = slice(h * g, (h + 1) * g)
                    rows = [torch.cat((x[i][prefix_table[0].long(), h].reshape(-1, d)[:kept], x[i][table[b].long(), h].reshape(-1, d)[:s + 1])).double().cpu() for x in (kp, vp)]
                    assert torch.equal(rows[0][:kept], k_out[i][h].double().cpu())
                    want = attend(q_rot[i, b, heads].double().cpu(), *rows, d ** -0.5, dtype)
                    near(out[i, b, heads], want[0], want[2], f"step {s}")
                    near_lse(lse[i, b, heads], want[1], want[3], f"step {s}, lse")
