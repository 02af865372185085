"""What h's rounding to bf16 on its way to 8 bits may cost, on the host (oracle/int8.py)."""
import numpy as np
import torch

from oracle import int8 as O


def test_rows_by_way_of_bf16_are_off_by_up_to_a_step():
    """bf16 is off by 2^-8 of a value, 127 / 256 of a step where it is the largest of its row, and 8 bits by half a step."""
    g = torch.Generator().manual_seed(0)
    h = torch.randn((400, 2816), generator=g, dtype=torch.float64)
    h *= torch.randn(h.shape, generator=g, dtype=torch.float64)              # a product of two, as silu(g) * u is
    q, scale = O.quantize(h.to(torch.bfloat16).float().numpy())
    step = scale.astype(np.float64)[:, None]
    off = np.abs(q * step - h.numpy()) / step
    bound = 0.5 + np.abs(h.numpy()) * O.U16 / step + 127 * 4 * O.U           # the quotient by a rounded inverse, as in the GPU tests
    assert (off <= bound).all() and (bound <= 1.01).all()
    assert off.max() > 0.75                                                   # more than half a step and a quarter
