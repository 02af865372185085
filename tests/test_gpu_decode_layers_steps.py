"""DecodeLayers on the GPU over many steps: a step that fails and is taken again, requests that are done and others in their seats,
steps without rows."""
import pytest
import torch

import paper_2411_11217_amd as M
from paper_2411_11217_amd import binding as B
from test_gpu_decode_layers import build

pytestmark = pytest.mark.gpu


def tokens(T, seed):
    return torch.randn((T, 256), generator=torch.Generator().manual_seed(seed)).cuda()


def i32(v):
    return torch.tensor(v, dtype=torch.int32).cuda()


def test_a_step_that_failed_can_be_taken_again(monkeypatch):
    _, _, _, one = build()
    _, _, _, other = build()
    real, calls = B.moe_post_attention, []

    def fails(*args, **kw):
        out = real(*args, **kw)
        calls.append(1)
        if len(calls) == 2:                                # the second layer's
            raise MemoryError
        return out

    for n, fresh in enumerate([[7, 0, 3], [1, 1, 1], [1, 1, 1], [1, 4, 1], [1, 1, 1]]):
        x = tokens(sum(fresh), n)
        want, _ = one.step(x, i32(fresh))
        calls.clear()
        monkeypatch.setattr(B, "moe_post_attention", fails)
        with pytest.raises(MemoryError):
            other.step(x, i32(fresh))
        monkeypatch.setattr(B, "moe_post_attention", real)
        got, _ = other.step(x, i32(fresh))
        torch.cuda.synchronize()
        assert torch.equal(got, want) and torch.equal(one.lengths, other.lengths) and torch.equal(one.free_head, other.free_head)
    assert other.status.tolist() == [0, 0, 0, 0]


def test_seats_and_pages_of_retired_requests_are_used_again():
    # a pool of 9 pages: three requests fill it, one is refused, two go, others come in their seats; what these get is what they get alone
    _, _, _, model = build(pool_pages=9)
    model.step(tokens(30, 1), i32([12, 10, 8]))            # three pages, three, two
    _, tables = model.step(tokens(8, 2), i32([1, 1, 6]))   # one page, none, two: none is left
    torch.cuda.synchronize()
    assert model.lengths.tolist() == [13, 11, 8] and model.status.tolist() == [2, 0, 0, 0] and tables.free_head.tolist() == [9]
    model.retire(torch.tensor([True, False, True]).cuda())
    torch.cuda.synchronize()
    assert model.lengths.tolist() == [0, 11, 0] and model.free_head.tolist() == [3]
    held = model.block_table[1, :3].tolist()
    assert sorted(held + model.free_pages[3:].tolist()) == list(range(9)) and (model.block_table[[0, 2]] == -1).all()
    model.status.zero_()
    _, _, _, fresh = build(pool_pages=30)
    a, _ = model.step(tokens(21, 3), i32([9, 0, 12]))      # all six pages
    b, _ = fresh.step(tokens(21, 3), i32([9, 0, 12]))
    torch.cuda.synchronize()
    assert model.status.tolist() == [0, 0, 0, 0] and model.lengths.tolist() == [9, 11, 12] and model.free_head.tolist() == [9] and torch.equal(a, b)


def test_steps_without_rows():
    _, _, _, model = build()
    out, _ = model.step(tokens(0, 1), i32([0, 0, 0]))
    assert out.shape == (0, 256)
    model.step(tokens(5, 1), i32([2, 0, 3]))
    out, tables = model.step(tokens(0, 1), i32([0, 0, 0]))
    torch.cuda.synchronize()
    assert out.shape == (0, 256) and model.lengths.tolist() == [2, 0, 3] and tables.row_start.tolist() == [0, 0, 0, 0]
    assert model.status.tolist() == [0, 0, 0, 0]
