"""DecodeLayers with 8-bit weights on the GPU: mixed steps of prompts and single tokens against the library's operators called one by one."""
import pytest
import torch

import paper_2411_11217_amd as M

pytestmark = pytest.mark.gpu
H, F, E, K, N_Q, N_KV, D, P, PAGE = 256, 512, 4, 2, 4, 2, 64, 4, 65536
WIDE = (N_Q + 2 * N_KV) * D


def build(n_layers=2, n_requests=3):
    g = torch.Generator().manual_seed(9)
    s = M.make_shape(1, H, F, E, K, "i8", PAGE)
    kv = M.make_kv_shape(N_Q, N_KV, D, P, 16, 60, "bf16")
    layers = []
    for _ in range(n_layers):
        dense = {n: torch.randn(shape, generator=g) * 0.06 for n, shape in dict(qkv=(WIDE, H), o=(H, N_Q * D), w1=(E, F, H), w3=(E, F, H), w2=(E, H, F)).items()}
        q = {}
        for n, w in dense.items():               # a weight's channels are rows like any others
            rows, scale = M.moe_quantize_i8(w.reshape(-1, w.shape[-1]).cuda())
            q[n] = (rows.view(w.shape).cpu(), scale.view(w.shape[:-1]))
        pw = M.PagedWeights(s, q["w1"][0], q["w3"][0], q["w2"][0])
        q_shape, o_shape = M.make_linear_shape(1, H, WIDE, PAGE, "i8"), M.make_linear_shape(1, N_Q * D, H, PAGE, "i8")
        n_q, n_o = M.linear_pages_required(q_shape), M.linear_pages_required(o_shape)
        pool = torch.zeros((pw.pool_pages + n_q + n_o, PAGE), dtype=torch.uint8)
        pool[:pw.pool_pages] = pw.pages_host
        q_table = torch.arange(pw.pool_pages, pw.pool_pages + n_q, dtype=torch.int32)
        o_table = torch.arange(pw.pool_pages + n_q, pw.pool_pages + n_q + n_o, dtype=torch.int32)
        M.linear_pack(q_shape, q["qkv"][0], q_table, pool)
        M.linear_pack(o_shape, q["o"][0], o_table, pool)
        gammas = [(1 + 0.1 * torch.randn(H, generator=g)).cuda() for _ in range(2)]
        Wr = (torch.randn((E, H), generator=g) * 0.1).to(torch.bfloat16).cuda()
        scales = M.LayerScales(q["qkv"][1], q["o"][1], M.ExpertScales(q["w1"][1], q["w3"][1], q["w2"][1]))
        layers.append(M.LayerWeights(pool.cuda(), q_table.cuda(), o_table.cuda(), pw.table_host.cuda(), Wr, gammas[0], gammas[1], scales=scales))
    freq = torch.tensor([1000.0 ** (-i / 32) for i in range(32)], dtype=torch.float64).cuda()
    return layers, freq, M.DecodeLayers(s, kv, layers, freq, n_requests)


def test_a_step_is_its_calls():
    """Each layer of each step again, through the single operators, on caches of their own."""
    layers, freq, model = build()
    s, kv = model.shape, model.kv
    caches = [(torch.zeros_like(k), torch.zeros_like(v)) for k, v in model.caches]
    g = torch.Generator().manual_seed(3)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    for fresh in ([7, 0, 3], [1, 5, 1], [1, 1, 1], [0, 0, 30]):
        T = sum(fresh)
        x = torch.randn((T, H), generator=g).cuda()
        out, tables = model.step(x, torch.tensor(fresh, dtype=torch.int32).cuda())
        seen = torch.where(tables.slots >= 0, tables.positions + 1, 0)
        hidden, delta = None, x
        q_shape, o_shape, st = M.make_linear_shape(T, H, WIDE, PAGE, "i8"), M.make_linear_shape(T, N_Q * D, H, PAGE, "i8"), s.with_tokens(T)
        for w, (kc, vc) in zip(layers, caches):
            hidden, _, q, scale = M.moe_add_rmsnorm_i8(hidden, delta, w.norm_attn, 1e-5, want_x=False)
            qkv = M.moe_linear_i8(q_shape, q, scale, w.qkv_table, w.page_pool, w.scales.qkv, status=status)
            queries = M.moe_qk_norm_rope(kv, qkv, freq, tables.positions, tables.slots, kc, vc)
            attn, _ = M.moe_attn_decode(kv, queries, seen, model.block_table, kc, vc, table_row=tables.request)
            q, scale = M.moe_quantize_i8(attn.view(T, N_Q * D))
            proj = M.moe_linear_i8(o_shape, q, scale, w.o_table, w.page_pool, w.scales.o, status=status)
            hidden, rows, q, scale = M.moe_add_rmsnorm_i8(hidden, proj, w.norm_moe, 1e-5)
            ids, weights, _ = M.moe_route(st.routed(), rows, w.Wr)
            p = M.moe_permute(st.routed(), ids, topk_w=weights)
            _, _, o = M.moe_expert_ffn_i8(st, q, scale, p["offsets"], w.page_table, w.page_pool, w.scales.experts, row_src=p["row_src"], row_w=p["row_w"], status=status)
            delta = M.moe_combine(st, o, p["row_of"])
        assert torch.equal(out, hidden + delta)
        assert model.status.tolist() == [0] * 4 and status[0] == 0
    assert model.lengths.tolist() == [7 + 1 + 1, 5 + 1, 3 + 1 + 1 + 30]


def test_prompts_at_once_and_token_by_token():
    """A prompt in one step, and the same tokens one by one: the calls around attention give a row the same bits in any company, so the first token, which
    attends to itself alone, is the same; later ones differ by the roundings of the attention's sums, which may turn a step of the 8 bits."""
    _, _, a = build()
    _, _, b = build()
    x = torch.randn((6, H), generator=torch.Generator().manual_seed(8)).cuda()
    at_once, _ = a.step(x, torch.tensor([0, 6, 0], dtype=torch.int32).cuda())
    one = [b.step(x[i:i + 1], torch.tensor([0, 1, 0], dtype=torch.int32).cuda())[0] for i in range(6)]
    assert torch.equal(one[0][0], at_once[0])
    assert a.lengths.tolist() == b.lengths.tolist() == [0, 6, 0]
    assert torch.isfinite(torch.cat(one)).all()


def test_a_step_without_rows():
    _, _, model = build()
    out, _ = model.step(torch.empty((0, H), device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, H) and model.lengths.tolist() == [0, 0, 0]
