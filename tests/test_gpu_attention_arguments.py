"""Calls of the attention over a paged cache at the ends of their arguments' ranges, on the GPU."""
import pytest
import torch

import paper_2411_11217_amd as M
from test_gpu_attention import Cache, attend_and_compare, i32, new_status, queries

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("head", [0, 3, 7])
def test_tables_of_a_step_without_requests_and_rows_hand_the_head_on(head):
    kv = M.make_kv_shape(1, 1, 32, 16, 4, 10, "bf16")
    status = new_status()
    step = M.KvStep(kv, 0, 0)
    step.buf.fill_(-7)                           # what a step's memory may hold from before
    M.moe_kv_assign(kv, i32([]), i32([]), i32(range(7)), i32([head]), torch.zeros((0, 4), dtype=torch.int32, device="cuda"), step=step, status=status)
    torch.cuda.synchronize()
    assert step.free_head.tolist() == [head] and step.row_start.tolist() == [0] and status.tolist() == [0, 0, 0, 0]


def test_norm_rope_of_more_rows_than_a_grid_has_threads_for():
    # 2^24 + 9 rows: 256 threads each would be more than 2^32
    T, D = 2 ** 24 + 9, 32
    kv = M.make_kv_shape(1, 1, D, 16, 1, T // 16 + 1, "bf16")
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.empty((T, 3 * D), dtype=torch.bfloat16, device="cuda").normal_(generator=g)
    k, v = (torch.zeros(kv.cache_shape, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    rows = torch.arange(T, dtype=torch.int32, device="cuda")
    q = M.moe_qk_norm_rope(kv, x, torch.zeros(0, dtype=torch.float64, device="cuda"), rows, rows, k, v)
    torch.cuda.synchronize()
    assert torch.equal(q[:, 0], x[:, :D])
    assert torch.equal(k.view(-1, D)[:T], x[:, D:2 * D]) and torch.equal(v.view(-1, D)[:T], x[:, 2 * D:])
    # and rotated, at both ends of every part of the rows
    freq = torch.tensor([0.3, 0.01, 0.002, 1e-4], dtype=torch.float64, device="cuda")
    q = M.moe_qk_norm_rope(kv, x, freq, rows, rows, k, v)
    at = torch.tensor([0, 1, 2 ** 23 - 1, 2 ** 23, 2 ** 24 - 1, 2 ** 24, T - 1], device="cuda")
    want = M.moe_qk_norm_rope(kv, x[at].contiguous(), freq, rows[at].contiguous(), torch.full((7,), -1, dtype=torch.int32, device="cuda"), k, v)
    torch.cuda.synchronize()
    assert torch.equal(q[at], want)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (2, 1), (3, 1), (8, 2), (5, 1), (8, 1)])
def test_rows_of_one_request_on_both_sides_of_sharing(n_q, n_kv, dtype):
    # groups whose rows share and groups whose rows do not, in turn: far apart under a window, a few long rows among short ones, all long
    lens = [900, 260]
    c = Cache(lens, n_kv, 64, 16, dtype, n_q)
    kv = M.make_kv_shape(n_q, n_kv, 64, 16, c.table.shape[1], c.k.shape[0], dtype)
    pack = 16 // (n_q // n_kv)
    seq, rows = [], []
    for n in range(45):
        long = n % (pack + 1)                              # of the group's rows
        seq += [10 + (7 * n + i) % 20 if i >= long else 850 - 13 * i for i in range(pack)] if n % 3 else [16 * (i + n % 5) + 3 for i in range(pack)]
        rows += [n % 2 if n % 3 == 0 else 0] * pack
    seq = [min(s, lens[b]) for s, b in zip(seq, rows)]
    q = queries(len(seq), kv, dtype, n_q + 1)
    for n in {len(seq), 64, 3 * pack, 61}:
        for window in (0, 24, 300):
            attend_and_compare(c, kv, q[:n], seq[:n], dtype, window=window, table_row=rows[:n], rows=range(0, n, 1 if n < 100 else 5), what=f"{n_q}/{n_kv} {dtype} {n} rows, window {window}")


@pytest.mark.parametrize("n_q,n_kv,lens", [(4, 1, [300, 300, 300, 640]), (4, 1, [640, 300, 300, 300]), (2, 1, [300] * 7 + [640]), (4, 1, [300, 300, 300, 640] * 40)])
def test_pages_between_the_windows_of_rows_that_share_are_not_followed(n_q, n_kv, lens):
    # rows of one request under a window: what no row sees may be gone from the block table
    c = Cache([640], n_kv, 64, 16, "bf16", 2)
    kv = M.make_kv_shape(n_q, n_kv, 64, 16, c.table.shape[1], c.k.shape[0], "bf16")
    q, rows = queries(len(lens), kv, "bf16", 3), [0] * len(lens)
    for gone in (-1, 2 ** 31 - 1):
        c.table[0, 19:21] = gone                           # tokens 304 to 335; the rows see 0 to 299 and 340 to 639
        attend_and_compare(c, kv, q, lens, "bf16", window=300, table_row=rows)
