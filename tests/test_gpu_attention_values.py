"""Attention on the GPU where single values decide: weights with all of their bits, infinite values."""
import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from test_gpu_attention import DT, HALF_STEP, Cache, f64, i32, queries
from util import say

pytestmark = pytest.mark.gpu
U = 2.0 ** -24                                   # half a step of float32, relative


# ---------------------------------------------------------------------------- weights

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("share", [False, True])
def test_attention_weights_have_all_bits_of_float32(dtype, share):
    """Two tokens with scores 0 and s, values A and -B with A close to exp(s) B: what is left is far smaller than either, so that its own rounding
    to bf16 hides nothing.  The arithmetic is off by: s is exact (one product that is not 0); exponent's factor and product, 2 U |s|; the exponential,
    2 U; so a weight by 5 U; the products are exact, their up to six sums off by 2 U each; the sum of the weights and its inverse 5 U, the last product U: 24 U of sum p |v| / sum p."""
    g = np.random.default_rng(1)
    D, R, heads = 64, 40, 4
    kv = M.make_kv_shape(heads, 1, D, 16, 1, R, dtype)
    s = torch.tensor(-g.uniform(0.05, 1.4, (R, heads)), dtype=torch.float32).to(torch.bfloat16).double().numpy()
    mantissas = np.arange(128, 256) / 128.0
    a, b = mantissas[:, None], mantissas[None, :] * 2.0 ** np.arange(0, 3)[:, None, None]      # A in [1, 2), B in [1, 8)
    q, k, v = np.zeros((R, heads, D)), np.zeros((R, 1, 16, D)), np.zeros((R, 1, 16, D))
    k[:, 0, 1, 0] = 1.0
    for r in range(R):
        for h in range(heads):
            q[r, h, 0] = s[r, h]
            best = np.argsort(np.abs(a - np.exp(s[r, h]) * b).ravel())[:D // heads]            # the closest pairs
            e, i, j = np.unravel_index(best, (3, 128, 128))
            v[r, 0, 0, h::heads], v[r, 0, 1, h::heads] = mantissas[i], -mantissas[j] * 2.0 ** e
    dev = [torch.tensor(x).to(DT[dtype]) for x in (q, k, v)]
    assert all(np.array_equal(f64(t), x) for t, x in zip(dev, (q, k, v)))
    order = torch.arange(R, dtype=torch.int32)
    row = order if share else None
    if share:                                    # four rows of one request: they share the columns of the products
        row = (order // 4) * 4
        k, v = k[row], v[row]
    out, _ = M.moe_attn_decode(kv, dev[0].cuda(), i32([2] * R), order.view(R, 1).cuda(), dev[1].cuda(), dev[2].cuda(), scale=1.0, table_row=None if row is None else row.cuda())
    torch.cuda.synchronize()
    p = np.exp(s)[..., None]
    v0, v1 = v[:, :, 0], v[:, :, 1]
    ref, size = (v0 + p * v1) / (1 + p), (np.abs(v0) + p * np.abs(v1)) / (1 + p)
    bound = 24 * U * size
    room = bound + HALF_STEP[dtype] * (np.abs(ref) + bound)
    worst = (np.abs(f64(out) - ref) / room).max()
    say(f"    {dtype} share={share}: {worst:.3f} of what is allowed")
    assert worst <= 1.0
