"""Calls of the attention over a paged cache at the ends of their arguments' ranges, on the GPU."""
import pytest
import torch

import paper_2411_11217_amd as M
from test_gpu_attention import i32, new_status

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
