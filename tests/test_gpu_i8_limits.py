"""The layer in 8-bit integers at the ends of what its calls take."""
import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import int8 as O

pytestmark = pytest.mark.gpu


def test_as_many_rows_as_the_call_counts():
    """T = 2^31 - 1, where T + 3 is no 32-bit number: four rows go to a block, and the last block has three."""
    T = 2 ** 31 - 1
    if torch.cuda.mem_get_info()[0] < 48 << 30:
        pytest.skip("34 GB of rows, whole numbers and scales")
    x = torch.empty((T, 4), dtype=torch.bfloat16, device="cuda").normal_(generator=torch.Generator(device="cuda").manual_seed(2))
    q, scale = M.moe_quantize_i8(x)
    rows = torch.cat([torch.arange(8), torch.arange(T - 9, T), torch.randint(0, T, (2000,), generator=torch.Generator().manual_seed(3))]).cuda()
    want_q, want_scale = O.quantize(x[rows].float().cpu().numpy())
    np.testing.assert_array_equal(q[rows].cpu().numpy(), want_q)
    np.testing.assert_array_equal(scale[rows].cpu().numpy(), want_scale)
