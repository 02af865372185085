"""Bad entries of page tables in the layer in 8-bit integers: read as page 0, and reported to whoever makes the call."""
import dataclasses

import pytest
import torch

import paper_2411_11217_amd as M
from test_gpu_i8 import Linear, layer_inputs
from test_gpu_i8_decode_layers import build

pytestmark = pytest.mark.gpu


def word(workspace):
    return workspace[:4].view(torch.int32).item()


def post_attention(T, H=512, K=768):
    """-> (call(o_table, page_table, workspace) -> (hidden_mid, y, status word), the good tables, slots of the pool)"""
    x, _, gamma, Wr = layer_inputs(T, H=H, seed=3)
    o = Linear(K, H, 16384)                      # pages of one tile: page_bytes of both have to be the same
    experts = x.pool.view(-1, 16384)             # the experts' pages of four tiles, one tile at a time
    table = (x.table[..., None] * 4 + torch.arange(4, dtype=torch.int32, device="cuda")).flatten(1)
    s = M.make_shape(T, H, x.F, x.E, x.k, "i8", 16384)
    gu, d = M.pages_required(s)
    whole = 4 * (M.pages_required(x.shape(T))[0])
    table = torch.cat([table[:, :gu], table[:, whole:whole + d]], 1).contiguous()
    pool = torch.cat([experts, o.pool])
    o_table = o.dev_table + experts.shape[0]
    o_proj = M.make_linear_shape(T, K, H, 16384, "i8")
    g = torch.Generator().manual_seed(T)
    hidden, attn = torch.randn((T, H), generator=g).cuda(), torch.randn((T, K), generator=g).to(torch.bfloat16).cuda()

    def call(o_table, page_table, workspace=None):
        mid, _, y, ws = M.moe_post_attention_i8(s, o_proj, attn, hidden, o_table, o.dev_scale, gamma, 1e-5, Wr, page_table, pool, x.dev, workspace=workspace)
        return mid, y, ws

    return call, o_table, table, pool.shape[0], M.binding.post_attention_i8_workspace_bytes(s, o_proj)


@pytest.mark.parametrize("T", [1, 40, 300, 1100])
def test_post_attention_reports_the_o_projection(T):
    """An entry of o_table outside the pool is in the workspace's status word, alone, beside one of the experts, and gone with the next call."""
    call, o_table, table, slots, need = post_attention(T)
    ws = torch.full((need,), 255, dtype=torch.uint8, device="cuda")
    mid, y, _ = call(o_table, table, ws)
    assert word(ws) == 0
    for entry, bad in ((0, -1), (o_table.numel() - 1, slots), (5, 2 ** 31 - 1)):
        broken = o_table.clone()
        broken[entry] = bad
        other, _, _ = call(broken, table, ws)
        assert word(ws) == 1 and torch.isfinite(other).all()
        keep = torch.arange(mid.shape[1]) // 128 != entry // 6           # 768 is six tiles of a column tile
        assert torch.equal(other[:, keep], mid[:, keep]) and not torch.equal(other, mid)
    experts = table.clone()
    experts[:, 1] = -7                           # whichever experts have rows
    again, _, _ = call(o_table, experts, ws)
    assert word(ws) == 1 and torch.equal(again, mid)
    call(broken, experts, ws)
    assert word(ws) == 1
    again, y2, _ = call(o_table, table, ws)
    assert word(ws) == 0 and torch.equal(again, mid) and torch.equal(y2, y)


def test_reports_of_a_captured_call():
    """Every replay says what its own tables hold."""
    call, o_table, table, slots, need = post_attention(70)
    ws, static = torch.zeros(need, dtype=torch.uint8, device="cuda"), o_table.clone()
    mid, y, _ = call(o_table, table)
    call(static, table, ws)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call(static, table, ws)
    for turn in range(4):
        static.copy_(o_table)
        if turn % 2:
            static[3] = slots + turn
        graph.replay()
        torch.cuda.synchronize()
        assert word(ws) == turn % 2
        if turn % 2 == 0:
            assert torch.equal(out[0], mid) and torch.equal(out[1], y)
        call(o_table, table)                     # eager work between the replays
        torch.cuda.synchronize()


def steps(model, fresh, seed):
    x = torch.randn((sum(fresh), 256), generator=torch.Generator().manual_seed(seed)).cuda()
    return model.step(x, torch.tensor(fresh, dtype=torch.int32).cuda())[0]


@pytest.mark.parametrize("field", ["o_table", "page_table", "qkv_table"])
@pytest.mark.parametrize("layer", [0, 1, 2])
def test_decode_layers_reports_its_weights(layer, field):
    """A bad entry of any table of any layer sets bit 0 of the model's status, which stays until the caller clears it."""
    layers, _, model = build(n_layers=3)
    want = [steps(model, f, n) for n, f in enumerate(([5, 0, 2], [1, 1, 1], [1, 40, 1], [1, 1, 1]))]
    assert model.status.tolist() == [0] * 4
    _, _, model = build(n_layers=3)
    good = getattr(layers[layer], field)
    bad = good.clone()
    bad.view(-1)[0] = -1                         # for the experts: of expert 0
    if field == "page_table":
        bad[:, 0] = -1
    assert torch.equal(steps(model, [5, 0, 2], 0), want[0]) and model.status.tolist() == [0] * 4
    model.layers[layer] = dataclasses.replace(model.layers[layer], **{field: bad})
    steps(model, [1, 1, 1], 1)
    assert model.status.tolist() == [1, 0, 0, 0]
    model.layers[layer] = dataclasses.replace(model.layers[layer], **{field: good})
    steps(model, [1, 40, 1], 2)
    steps(model, [0, 0, 0], 2)
    assert model.status.tolist() == [1, 0, 0, 0]
    model.status.zero_()
    steps(model, [1, 1, 1], 3)
    assert model.status.tolist() == [0] * 4


def test_decode_layers_status_holds_no_clock():
    """A QKV launch of more than 256 blocks reports the clock that it saw: not as a status of the model, whose words 1 to 3 stay zero."""
    layers, _, model = build(n_layers=1)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    T = 20000
    rows, scale = torch.ones((T, 256), dtype=torch.int8, device="cuda"), torch.ones(T, device="cuda")
    M.moe_linear_i8(M.make_linear_shape(T, 256, 512, 65536, "i8"), rows, scale, layers[0].qkv_table, layers[0].page_pool, layers[0].scales.qkv, status=status)
    assert status[0] == 0 and status[3] > 100    # so a step of this size has it too
    model.step(torch.randn((T, 256), device="cuda"), torch.tensor([1, 1, 1], dtype=torch.int32).cuda())      # rows behind the third belong to no request
    assert model.status.tolist() == [0] * 4
