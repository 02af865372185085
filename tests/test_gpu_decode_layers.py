"""DecodeLayers on the GPU: prompts and single tokens of several requests in mixed steps, each stage of each layer against the
oracle on the GPU's own inputs (a rounding flip must not cascade), and the same tokens in other steps."""
import numpy as np
import pytest
import torch

import oracle
import paper_2411_11217_amd as M
from moe_workloads import MoEConfig
from oracle import attention, dense
from paper_2411_11217_amd import binding as B
from util import Case, assert_close, assert_h_close, say

pytestmark = pytest.mark.gpu


def bits(t):
    return t.cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


N_Q, N_KV, D, P = 6, 2, 64, 4


def build(pool_pages=60, width=16, n_layers=2, n_requests=3, window=0):
    cfg = MoEConfig("decode", "bf16", T=1, H=256, F=384, E=4, k=2, page_bytes=64 * 1024, seed=41)
    case = Case(cfg)
    s = case.shape
    kv = M.make_kv_shape(N_Q, N_KV, D, P, width, pool_pages, "bf16")
    o_shape, q_shape = M.make_linear_shape(1, N_Q * D, s.H, s.page_bytes), M.make_linear_shape(1, s.H, (N_Q + 2 * N_KV) * D, s.page_bytes)
    n_exp, n_o, n_q = case.pw.pool_pages, M.linear_pages_required(o_shape), M.linear_pages_required(q_shape)
    layers, dense_weights = [], []
    for i in range(n_layers):
        g = torch.Generator().manual_seed(100 + i)
        pool = torch.zeros((n_exp + n_o + n_q, s.page_bytes), dtype=torch.uint8)
        pool[:n_exp] = case.pw.pages_dev.cpu()
        o_table, q_table = torch.arange(n_exp, n_exp + n_o, dtype=torch.int32), torch.arange(n_exp + n_o, n_exp + n_o + n_q, dtype=torch.int32)
        Wo, Wqkv = ((torch.randn(n, generator=g) * 0.06).to(torch.bfloat16) for n in ((s.H, N_Q * D), ((N_Q + 2 * N_KV) * D, s.H)))
        M.linear_pack(o_shape, Wo, o_table, pool)
        M.linear_pack(q_shape, Wqkv, q_table, pool)
        gammas = [(1.0 + 0.1 * torch.randn(n, generator=g)).cuda() for n in (s.H, s.H, D, D)]
        layers.append(M.LayerWeights(pool.cuda(), q_table.cuda(), o_table.cuda(), case.pw.table_dev, case.Wr, gammas[0], gammas[1], None, gammas[2], gammas[3]))
        dense_weights.append((Wo, Wqkv))
    inv_freq = torch.tensor([1000.0 ** (-i / 32) for i in range(32)], dtype=torch.float64).cuda()
    return case, layers, dense_weights, M.DecodeLayers(s, kv, layers, inv_freq, n_requests, window=window)


def test_every_stage_of_mixed_steps_matches_the_oracle(monkeypatch):
    case, layers, dense_weights, model = build()
    seen = []                                              # (call, its inputs and outputs) of a step

    def record(name):
        real = getattr(B, name)

        def call(*args, **kw):
            out = real(*args, **kw)
            seen.append((name, args, kw, out))
            return out
        monkeypatch.setattr(B, name, call)

    for name in ("moe_pre_attention", "moe_qk_norm_rope", "moe_attn_decode", "moe_post_attention"):
        record(name)
    g = torch.Generator().manual_seed(1)
    history = [[(np.zeros((0, N_KV, D)), np.zeros((0, N_KV, D))) for _ in range(3)] for _ in layers]
    lengths = np.zeros(3, np.int64)
    for fresh in ([7, 0, 3], [1, 5, 1], [1, 1, 1], [1, 1, 0]):
        seen.clear()
        T = sum(fresh)
        x = torch.randn((T, 256), generator=g)
        out, tables = model.step(x.cuda(), torch.tensor(fresh, dtype=torch.int32).cuda())
        torch.cuda.synchronize()
        lengths += fresh
        assert model.status.tolist() == [0, 0, 0, 0] and model.lengths.tolist() == lengths.tolist()
        pos, req = tables.positions.cpu().numpy(), tables.request.cpu().numpy()
        assert len(seen) == 4 * len(layers)
        residual = x.double().numpy()                      # what enters the layer: hidden + delta
        for i, w in enumerate(layers):
            (_, _, _, (hidden, x_norm, qkv, _)), (_, _, _, q), (_, _, _, (attn, _)), (_, _, _, (mid, x_moe, y, _)) = seen[4 * i:4 * i + 4]
            Wo, Wqkv = dense_weights[i]
            assert_close(hidden.cpu().numpy(), residual, "f32", "residual")
            _, xn = dense.add_rmsnorm(None, hidden.cpu().numpy(), w.norm_attn.cpu().numpy(), model.eps)
            assert_h_close(x_norm.float().cpu().numpy(), dense.bf16_bits_to_f64(xn), "bf16", "norm")
            assert_close(qkv.cpu().numpy(), dense.linear(bits(x_norm), bits(Wqkv)), "bf16", "QKV projection")
            heads = qkv.cpu().double().numpy().reshape(T, -1, D)
            inv_freq = model.inv_freq.cpu().numpy()
            for got, sl, gamma in ((q, slice(0, N_Q), w.q_gamma), (None, slice(N_Q, N_Q + N_KV), w.k_gamma)):
                ref, bound = attention.qk_norm_rope(heads[:, sl], gamma.cpu().double().numpy(), model.eps, inv_freq, pos, False)
                if got is None:
                    slots = tables.slots.cpu().numpy()
                    got = k_new = model.caches[i][0].cpu()[slots // P, :, slots % P]
                assert (np.abs(got.cpu().double().numpy() - ref) <= bound + 2.0 ** -8 * (np.abs(ref) + bound)).all()
            v_new = model.caches[i][1].cpu()[slots // P, :, slots % P]
            assert torch.equal(v_new, qkv.cpu().view(T, -1, D)[:, N_Q + N_KV:].to(torch.bfloat16))
            for b in range(3):
                mine = req == b
                history[i][b] = tuple(np.concatenate([h, n.double().numpy()[mine]]) for h, n in zip(history[i][b], (k_new, v_new)))
            for r in range(T):
                ks, vs = history[i][req[r]]
                for h in range(N_KV):
                    hs = slice(h * 3, h * 3 + 3)
                    ref, _, bound, _ = attention.attend(q[r, hs].cpu().double().numpy(), ks[:pos[r] + 1, h], vs[:pos[r] + 1, h], D ** -0.5, True)
                    assert (np.abs(attn[r, hs].cpu().double().numpy() - ref) <= bound + 2.0 ** -8 * (np.abs(ref) + bound)).all()
            o = dense.linear(bits(attn.view(T, -1)), bits(Wo))
            assert_close(mid.cpu().numpy(), hidden.cpu().double().numpy() + o, "bf16", "O projection + residual")
            v = case.view
            ref = oracle.layer(bits(x_moe), v["Wr"], v["W1"], v["W3"], v["W2"], 2, 1)
            clear = ref["gap_next"] >= 1e-4
            assert_close(y.cpu().numpy()[clear], ref["y"][clear], "bf16", "MoE layer")
            residual = mid.cpu().double().numpy() + y.cpu().double().numpy()
        assert_close(out.cpu().numpy(), residual, "f32", "output")
        say(f"    step {fresh}: all stages")


def test_prompt_at_once_equals_token_by_token():
    # one request's seven tokens in one step, and one by one beside another request: the same results up to the order of sums
    g = torch.Generator().manual_seed(2)
    x = torch.randn((7, 256), generator=g).cuda()
    _, _, _, a = build()
    at_once, _ = a.step(x, torch.tensor([0, 7, 0], dtype=torch.int32).cuda())
    _, _, _, b = build()
    other = torch.randn((7, 256), generator=g).cuda()
    rows = []
    for t in range(7):
        out, _ = b.step(torch.stack([other[t], x[t]]), torch.tensor([1, 1, 0], dtype=torch.int32).cuda())
        rows.append(out[1])
    torch.cuda.synchronize()
    err = (torch.stack(rows) - at_once).abs().max().item()
    say(f"    max difference {err:.3e}")
    # values of up to about 5; two layers whose bf16 intermediates may differ by a step (2^-7 of the value) where a sum fell on the other side
    assert err <= 0.1 and a.lengths.tolist() == [0, 7, 0] and b.lengths.tolist() == [7, 7, 0]


def test_requests_that_find_no_pages_are_refused_and_the_others_go_on():
    _, _, _, model = build(pool_pages=5)
    x = torch.randn((14, 256), generator=torch.Generator().manual_seed(3)).cuda()
    model.step(x[:9], torch.tensor([4, 4, 1], dtype=torch.int32).cuda())                 # three pages
    _, tables = model.step(x, torch.tensor([4, 9, 1], dtype=torch.int32).cuda())         # one page, three (one is left), none needed
    torch.cuda.synchronize()
    assert model.status.tolist() == [2, 0, 0, 0] and model.lengths.tolist() == [8, 4, 2] and tables.free_head.tolist() == [4]
    slots = tables.slots.cpu()
    assert (slots[4:13] == -1).all() and (slots[:4] >= 0).all() and slots[13] >= 0
