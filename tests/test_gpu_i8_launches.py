"""The kernels of the layer in 8-bit integers that only larger sizes take, each named by the host's formulas (tests/util.py): the linear map's wide blocks and its blocks with teams, the experts
of weights that come with the non-temporal hint, rows in 8 bits read and written with it."""
import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import int8 as O
from test_gpu_i8 import Experts, Linear, bf16_values, check_quantized, rows_of
from util import i8_expert_launches, i8_linear_launch

pytestmark = pytest.mark.gpu

# ---------------------------------------------------------------------------- the linear map

WIDE = ("ffn_gemm", 1, 2, 256, 0)                # 256 rows x 256 columns


def check_rows(lin, q, scale, out, rows):
    lin.check(q[rows], scale[rows], out[rows.cuda()])


@pytest.mark.parametrize("K,N", [(256, 20480), (256, 20608), (1280, 16512)])
def test_linear_wide_blocks(K, N):
    """Even and odd numbers of page tiles (half of the last block's columns are none), every height of a last row tile.  Each row has the bits of a call of its own, which takes another kernel."""
    lin = Linear(K, N, 65536)
    q, scale = lin.rows(2100)
    few = lin.run(q[:40], scale[:40])
    assert i8_linear_launch(40, K, N) != WIDE
    for T in (1792, 1793, 1808, 1809, 1824, 1825, 1888, 1985, 2047, 2100):
        assert i8_linear_launch(T, K, N) == WIDE
        out = lin.run(q[:T], scale[:T])
        assert torch.equal(out[:40], few) and torch.equal(out[T - 35:], lin.run(q[T - 35:T], scale[T - 35:T]))
        check_rows(lin, q, scale, out, torch.cat([torch.arange(0, 1792, 97), torch.arange(1785, T)[-64:]]))


def test_linear_wide_blocks_bad_pages():
    """Entries of the first, a middle and the last column tile, of which the last shares its block with none."""
    lin, T = Linear(256, 20608, 16384), 1825     # two pages to a column tile
    assert i8_linear_launch(T, 256, 20608) == WIDE
    q, scale = lin.rows(T)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    want = lin.run(q, scale, status=status)
    assert status[0] == 0
    good = lin.dev_table
    for entry, bad in ((0, -1), (161, 2 ** 31 - 1), (321, lin.pool.shape[0])):
        lin.dev_table = good.clone()
        lin.dev_table[entry] = bad
        out = lin.run(q, scale, status=status)
        keep = torch.arange(20608) // 128 != entry // 2
        assert status[0].item() == 1 and torch.equal(out[:, keep], want[:, keep]) and not torch.equal(out, want)
        status.zero_()


@pytest.mark.parametrize("K,N,T,kernel", [
    (256, 12288, 72, (8, 4, 1, 2, 4, 1)), (1024, 9728, 96, (8, 4, 1, 2, 4, 1)),                                  # 128 rows, one team
    (4096, 5120, 300, (8, 4, 1, 2, 4, 2)), (4352, 2816, 545, (8, 4, 1, 2, 4, 2)),                                # two teams, the second with more steps
    (2048, 9600, 100, (4, 5, 1, 1, 4, 2)), (2304, 384, 3001, (4, 5, 1, 1, 4, 2)), (256, 384, 3001, (4, 5, 1, 1, 4, 1)),      # 80 columns
    (2048, 12288, 100, (4, 6, 1, 1, 4, 2)), (4352, 768, 1601, (4, 6, 1, 1, 4, 2)), (512, 768, 1601, (4, 6, 1, 1, 4, 1)),     # 96
    (2304, 512, 3001, (4, 8, 1, 1, 4, 2)), (2304, 128, 3001, (4, 2, 1, 2, 4, 4)), (2304, 256, 3001, (4, 4, 1, 1, 4, 4)),
    (2560, 256, 1030, (2, 3, 1, 1, 4, 4)), (2816, 128, 500, (2, 1, 1, 2, 4, 8)), (1792, 256, 900, (2, 2, 1, 2, 4, 4))])
def test_linear_blocks_for_few_rows(K, N, T, kernel):
    lin = Linear(K, N, 65536)
    assert i8_linear_launch(T, K, N) == ("ffn_rows", 1) + kernel
    q, scale = lin.rows(T)
    out = lin.run(q, scale)
    check_rows(lin, q, scale, out, torch.arange(T) if T <= 600 else torch.cat([torch.arange(0, T, 13), torch.arange(T - 70, T)]))
    assert torch.equal(out[:7], lin.run(q[:7], scale[:7])) and torch.equal(out[T - 20:], lin.run(q[T - 20:], scale[T - 20:]))


# ---------------------------------------------------------------------------- the experts

def first_rows(x, got, row_src, n=3):
    at = [int((row_src == t).nonzero()) for t in range(n)]
    return [t.cpu()[at] for t in got]


@pytest.mark.parametrize("H,F,calls", [
    # 201 MB: weights and h with the hint for experts of one row tile
    (2048, 4096, [(4, ("ffn_thin", 0, 2), ("ffn_thin", 1, 1), 1), (160, ("ffn_rows", 0, 4, 8, 1, 1, 4, 1), ("ffn_rows", 1, 4, 4, 1, 1, 4, 1), 1),
                  (300, ("ffn_rows", 0, 4, 8, 1, 1, 4, 1), ("ffn_rows", 1, 4, 4, 1, 1, 4, 1), 1), (700, ("ffn_rows", 0, 8, 8, 1, 1, 2, 1), ("ffn_rows", 1, 8, 4, 1, 1, 4, 1), 1),
                  (1400, ("ffn_gemm", 0, 2, 256, 0), ("ffn_gemm", 1, 1, 256, 1), 1), (3000, ("ffn_gemm", 0, 2, 256, 0), ("ffn_gemm", 1, 1, 256, 0), 0)]),
    # 604 MB: h with the hint for all experts
    (4096, 6144, [(4, ("ffn_thin", 0, 2), ("ffn_thin", 1, 1), 2), (160, ("ffn_rows", 0, 4, 8, 1, 1, 4, 1), ("ffn_rows", 1, 4, 8, 1, 1, 4, 1), 2),
                  (560, ("ffn_rows", 0, 8, 7, 1, 1, 2, 1), ("ffn_rows", 1, 8, 8, 1, 1, 4, 1), 2), (1400, ("ffn_gemm", 0, 2, 256, 1), ("ffn_gemm", 1, 1, 256, 0), 2),
                  (2400, ("ffn_gemm", 0, 2, 256, 0), ("ffn_gemm", 1, 2, 256, 1), 0)])])
def test_experts_whose_weights_come_with_the_hint(H, F, calls):
    """The last call has no hint.  Experts of one and of several row tiles in every launch but the first; a token's row has the same bits in all of them."""
    x = Experts(H, F, 8, 1, 524288)
    T = calls[-1][0]
    q, scale = x.rows(T)
    logits = torch.randn((T, 8), generator=x.g)
    logits[:, 0] += 1.5
    ids = logits.argmax(1, keepdim=True)
    ids[:3] = torch.tensor([[0], [1], [0]])
    first = None
    for T, gate, down, stream in calls:
        assert i8_expert_launches(T, H, F, 8, 1) == (gate, down, stream)
        offsets, row_src, row_w = x.routing(T, ids[:T])
        rows = (offsets[1:] - offsets[:-1]).tolist()
        tile = {"ffn_thin": 16, "ffn_rows": 16 * gate[2], "ffn_gemm": 256}[gate[0]]
        assert T == 4 or (max(rows) > tile and any(0 < n <= tile for n in rows))
        row_w[[int((row_src == t).nonzero()) for t in range(3)]] = 0.75
        got = x.run(T, q[:T], scale[:T], offsets, row_src, row_w)
        x.check(q[:T], scale[:T], offsets, row_src, row_w, got, some=3)
        mine = first_rows(x, got, row_src)
        first = first or mine
        assert all(torch.equal(a, b) for a, b in zip(first, mine)), T


@pytest.mark.parametrize("H,F,E", [(2048, 512, 64), (1024, 1024, 64), (512, 14336, 8), (512, 28672, 4), (512, 33024, 4)])
@pytest.mark.parametrize("each", [20, 130])
def test_rows_of_h_written_past_the_caches(H, F, E, each):
    """Every number of wavefronts to a row of h, and rows that are too long for registers."""
    x, T = Experts(H, F, E, 1, 65536), each * E
    assert i8_expert_launches(T, H, F, E, 1)[2] == 1
    q, scale = x.rows(T)
    offsets, row_src, row_w = x.routing(T)
    x.check(q, scale, offsets, row_src, row_w, x.run(T, q, scale, offsets, row_src, row_w), some=2)


@pytest.mark.parametrize("T", [4, 300, 1400])
def test_experts_bad_pages_with_the_hint(T):
    x = Experts(2048, 4096, 8, 1, 65536)
    assert i8_expert_launches(T, 2048, 4096, 8, 1)[2] == 1
    q, scale = x.rows(T)
    offsets, row_src, row_w = x.routing(T)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    want = x.run(T, q, scale, offsets, row_src, row_w, status=status)
    assert status[0] == 0
    e = int((offsets[1:] - offsets[:-1]).argmax())
    other = torch.ones(T, dtype=torch.bool)
    other[int(offsets[e]):int(offsets[e + 1])] = False
    good = x.table
    for entry, bad in ((0, -1), (good.shape[1] - 1, x.pool.shape[0])):
        x.table = good.clone()
        x.table[e, entry] = bad
        got = x.run(T, q, scale, offsets, row_src, row_w, status=status)
        assert status[0].item() == 1 and all(torch.equal(a.cpu()[other], b.cpu()[other]) for a, b in zip(want, got))
        status.zero_()


def test_gate_up_blocks_of_128_rows_and_128_features():
    x, T = Experts(512, 4096, 8, 1, 65536), 480
    assert i8_expert_launches(T, 512, 4096, 8, 1) == (("ffn_rows", 0, 8, 8, 1, 1, 2, 1), ("ffn_rows", 1, 8, 4, 1, 1, 4, 1), 0)
    q, scale = x.rows(T)
    for ids in (None, torch.arange(T)[:, None] % 8, torch.zeros((T, 1), dtype=torch.int64)):
        offsets, row_src, row_w = x.routing(T, ids)
        x.check(q, scale, offsets, row_src, row_w, x.run(T, q, scale, offsets, row_src, row_w), some=40)


# ---------------------------------------------------------------------------- rows in 8 bits, norm, combine

@pytest.mark.parametrize("N,dtype", [(n, d) for n in (64, 252, 512, 516, 2044, 4096, 4100, 8192, 16380, 16384, 20480, 33000) for d in ("bf16", "f32")])
def test_quantize_rows_that_exceed_the_caches(N, dtype):
    """More than 16 MiB in all: the loads with the hint, for every number of wavefronts to a row."""
    T = (24 << 20) // (N * (3 if dtype == "bf16" else 5)) + 3
    x = torch.empty((T, N), device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(N)).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    q, scale = M.moe_quantize_i8(x)
    rows = torch.cat([torch.arange(0, T, max(1, T // 64)), torch.arange(T - 3, T)]).cuda()
    check_quantized(x[rows].cpu(), q[rows], scale[rows])
    some = slice(T // 2, T // 2 + 50)
    alone = M.moe_quantize_i8(x[some])
    assert torch.equal(alone[0], q[some]) and torch.equal(alone[1], scale[some])


@pytest.mark.parametrize("H", [128, 260, 1028, 4096, 6144, 8192])
def test_norm_rows_are_their_own(H):
    """Above 256 MiB in all the loads have the hint: a row's bits are those that it has alone."""
    T = (260 << 20) // (13 * H) + 5
    g = torch.Generator(device="cuda").manual_seed(H)
    hidden, delta = (torch.empty((T, H), device="cuda").normal_(generator=g) for _ in range(2))
    gamma = 1 + 0.2 * torch.empty(H, device="cuda").normal_(generator=g)
    whole = M.moe_add_rmsnorm_i8(hidden, delta, gamma, 1e-5)
    for rows in (slice(0, 70), slice(T // 2, T // 2 + 300), slice(T - 1, T)):
        part = M.moe_add_rmsnorm_i8(hidden[rows], delta[rows], gamma, 1e-5)
        assert all(torch.equal(a, b[rows]) for a, b in zip(part, whole))


@pytest.mark.parametrize("T,H,k,E", [(1, 256, 1, 1), (7, 512, 3, 5), (300, 1280, 8, 64), (33, 4096, 2, 8)])
def test_combine_of_bf16_rows_with_weights(T, H, k, E):
    """Rows times their weights, added in the order of the slots: each a fused product and sum."""
    g = torch.Generator().manual_seed(T)
    s = M.make_shape(T, H, 256, E, k, "i8", 65536)
    out, w = torch.randn((T * k, H), generator=g).to(torch.bfloat16), torch.rand((T, k), generator=g)
    row_of = torch.randperm(T * k, generator=g).to(torch.int32)
    y = M.moe_combine(s, out.cuda(), row_of.cuda(), w.cuda()).cpu().double().numpy()
    terms = bf16_values(out)[row_of.numpy()].reshape(T, k, H).astype(np.float64) * w.numpy().astype(np.float64)[..., None]
    assert (np.abs(y - terms.sum(axis=1)) <= np.abs(terms).sum(axis=1) * k * O.U).all()
    plain = M.moe_combine(s, out.cuda(), row_of.cuda()).cpu().double().numpy()
    values = bf16_values(out)[row_of.numpy()].reshape(T, k, H).astype(np.float64)
    assert (np.abs(plain - values.sum(axis=1)) <= np.abs(values).sum(axis=1) * k * O.U).all()
