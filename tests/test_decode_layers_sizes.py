"""Sizes that the norms of DecodeLayers do not take are refused when the layers are made, with bf16 and with 8-bit weights."""
import pytest
import torch

import paper_2411_11217_amd as M


def make(H, dtype, eps=1e-5):
    kv = M.make_kv_shape(4, 1, 64, 4, 6, 14, "bf16")
    scales = M.LayerScales(None, None, None) if dtype == "i8" else None
    return M.DecodeLayers(M.make_shape(1, H, 512, 4, 2, dtype, 65536), kv, [M.LayerWeights(*[None] * 7, scales=scales)], torch.zeros(16, dtype=torch.float64), 2, eps=eps, device="cpu")


@pytest.mark.parametrize("dtype", ["bf16", "i8"])
def test_rows_that_are_too_long_for_the_norm(dtype):
    make(8192, dtype)
    with pytest.raises(M.MoEError):
        make(8448, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "i8"])
@pytest.mark.parametrize("eps", [-1e-5, float("nan")])
def test_an_epsilon_that_the_norm_refuses(dtype, eps):
    make(256, dtype, 0.0)
    with pytest.raises(M.MoEError):
        make(256, dtype, eps)
