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
