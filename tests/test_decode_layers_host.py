"""What DecodeLayers keeps from step to step, on the host: its calls of the library are replaced by stand-ins on CPU tensors (the
tables by the oracle's), so that a step can fail at any of them."""
import types

import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import attention
from paper_2411_11217_amd import binding as B

H, P, WIDTH, POOL = 256, 4, 6, 14
CALLS = ("moe_kv_assign", "moe_pre_attention", "moe_qk_norm_rope", "moe_attn_decode", "moe_post_attention")


class Library:
    """Counts its calls, and fails at the one it is told to."""

    def __init__(self, monkeypatch):
        self.calls, self.fails = [], None
        for name in CALLS:
            monkeypatch.setattr(B, name, self.entry(name))
        monkeypatch.setattr(B, "AttnWorkspace", lambda kv, R, device: types.SimpleNamespace(buf=torch.zeros(B.attn_workspace_bytes(kv, R), dtype=torch.uint8)))

    def entry(self, name):
        def call(*args, **kw):
            self.calls.append(name)
            out = getattr(self, name)(*args, **kw)         # what was enqueued before an error has been done
            if self.fails is not None and len(self.calls) == self.fails:
                raise B.MoEError(B.ERR_INVALID_ARG, name)
            return out
        return call

    def moe_kv_assign(self, kv, cached, fresh, free_pages, free_head, block_table, step, status):
        outs = [getattr(step, n) for n in ("seq_len", "row_start", "positions", "slots", "request", "free_head")]
        if any(i.data_ptr() == o.data_ptr() for i in (cached, fresh, free_pages, free_head) for o in outs):
            raise B.MoEError(B.ERR_INVALID_ARG, "moe_kv_assign: an output is an input")
        r = attention.assign(kv.page_tokens, kv.max_pages, kv.pool_pages, step.T, cached.numpy(), fresh.numpy(), free_pages.numpy(), int(free_head), block_table.numpy())
        for o, n in zip(outs, ("seq_len", "row_start", "positions", "slots", "request", "free_head")):
            o.copy_(torch.from_numpy(r[n]))
        block_table.copy_(torch.from_numpy(r["block_table"]))
        status[0] |= r["status"]

    def moe_pre_attention(self, qkv_proj, hidden, delta, *rest, want_bf16):
        hidden = delta if hidden is None else hidden + delta
        return hidden, None, hidden[:, :192], None

    def moe_qk_norm_rope(self, kv, qkv, inv_freq, positions, slots, k_cache, v_cache, *rest, status):
        for r, s in enumerate(slots.tolist()):
            if s >= 0:
                k_cache[s // P, 0, s % P], v_cache[s // P, 0, s % P] = qkv[r, 128:160].bfloat16(), qkv[r, 160:192].bfloat16()
        return qkv[:, :128].bfloat16().view(-1, 4, 32)

    def moe_attn_decode(self, kv, q, seen, block_table, k_cache, v_cache, window, table_row, workspace, status):
        out = torch.zeros_like(q)
        for r, n in enumerate(seen.tolist()):
            t = torch.arange(n)
            if n:
                out[r] = (q[r] + v_cache[block_table[table_row[r]].long()[t // P], 0, t % P].float().sum(0)).bfloat16()
        return out, None

    def moe_post_attention(self, s, o_proj, attn, hidden, *rest, bias):
        return hidden, None, 0.5 * attn.float().repeat(1, H // 128), None


def build(n_layers=2, n_requests=3, dtype="bf16", n_q=4, H=H, layer_dtype="bf16", page_bytes=64 * 1024):
    kv = M.make_kv_shape(n_q, 1, 32, P, WIDTH, POOL, dtype)
    s = M.make_shape(1, H, 384, 4, 2, layer_dtype, page_bytes)
    layers = [M.LayerWeights(*[None] * 7) for _ in range(n_layers)]
    return M.DecodeLayers(s, kv, layers, torch.zeros(16, dtype=torch.float64), n_requests, device="cpu")


def kept(model):
    return [t.clone() for t in (model.lengths, model.free_head, model.block_table, model.free_pages, model.status)]


def tokens(T, seed):
    return torch.randn((T, H), generator=torch.Generator().manual_seed(seed))


def i32(v):
    return torch.tensor(v, dtype=torch.int32)


STEPS = ([2, 0, 3], [1, 3, 1], [1, 1, 1], [1, 1, 1], [3, 0, 0], [1, 1, 1], [0, 1, 0])


@pytest.mark.parametrize("fails", range(1, 10))
def test_a_step_that_fails_leaves_the_requests_as_they_were(fails, monkeypatch):
    # every step once with an error at the `fails`-th call of nine, once more at the next, then well: as a model that never failed
    lib = Library(monkeypatch)
    one, other = build(), build()
    for n, fresh in enumerate(STEPS):
        x = tokens(sum(fresh), n)
        want, _ = one.step(x, i32(fresh))
        for at in (fails, fails % 9 + 1):
            before = kept(other)
            lib.calls.clear()
            lib.fails = at
            with pytest.raises(M.MoEError, match=CALLS[0 if at == 1 else (at - 2) % 4 + 1]):
                other.step(x, i32(fresh))
            assert len(lib.calls) == at and torch.equal(before[0], other.lengths) and torch.equal(before[1], other.free_head)
        lib.fails = None
        got, tables = other.step(x, i32(fresh))
        assert torch.equal(got, want) and all(torch.equal(a, b) for a, b in zip(kept(one), kept(other)))
        assert tables.seq_len.data_ptr() == other.lengths.data_ptr()


def test_a_step_whose_last_sum_fails_leaves_the_requests_as_they_were(monkeypatch):
    lib = Library(monkeypatch)
    model = build(n_layers=1)
    model.step(tokens(3, 0), i32([1, 1, 1]))
    before = kept(model)
    whole = Library.moe_post_attention
    monkeypatch.setattr(Library, "moe_post_attention", lambda *a, **kw: (a[4], None, torch.zeros(7, 3), None))
    with pytest.raises(RuntimeError):
        model.step(tokens(3, 1), i32([1, 1, 1]))
    assert torch.equal(before[0], model.lengths) and torch.equal(before[1], model.free_head) and lib.fails is None
    monkeypatch.setattr(Library, "moe_post_attention", whole)
    model.step(tokens(3, 1), i32([1, 1, 1]))
    assert model.lengths.tolist() == [2, 2, 2]


def test_what_no_step_could_take_is_refused_when_the_layers_are_made(monkeypatch):
    monkeypatch.setattr(torch, "empty", lambda *a, **kw: pytest.fail("memory before the checks"))
    for kw in (dict(dtype="f32"), dict(layer_dtype="f32")):
        with pytest.raises(ValueError, match="bf16"):
            build(**kw)
    for kw in (dict(n_q=5), dict(n_q=0), dict(H=200), dict(page_bytes=1000), dict(n_requests=4097)):        # 160 values for the O projection, no heads, ..
        with pytest.raises((ValueError, M.MoEError)):
            build(**kw)


# ---------------------------------------------------------------------------- requests that are done

def pages_are_whole(model):
    """Every page of the pool is held by one request or free, once; behind a request's pages its row is of no concern."""
    held = [p for b, n in enumerate(model.lengths.tolist()) for p in model.block_table[b, :-(-n // P)].tolist()]
    assert sorted(held + model.free_pages[int(model.free_head):].tolist()) == list(range(POOL))
    assert model.free_pages.shape == (POOL,) and model.free_head.dtype is model.lengths.dtype is model.free_pages.dtype is torch.int32


def test_pages_of_retired_requests_are_used_again(monkeypatch):
    # a loop that takes several times the pool: seats are vacated at random, refusals included, and every request's outputs are those of a model that has had no other
    Library(monkeypatch)
    g = np.random.default_rng(3)
    model, alone, taken, refused = build(), [build(n_requests=1) for _ in range(3)], 0, 0
    for n in range(120):
        fresh = g.integers(0, 4, 3)
        before, x = model.lengths.clone(), tokens(int(fresh.sum()), n)
        out, tables = model.step(x, i32(fresh.tolist()))
        pages_are_whole(model)
        for b in range(3):
            grown = int(model.lengths[b] - before[b])
            assert grown in (0, fresh[b])
            refused += grown < fresh[b]
            if grown:
                rows = tables.request == b
                want, _ = alone[b].step(x[rows], i32([grown]))
                assert torch.equal(out[rows], want)
        done = torch.tensor(g.random(3) < 0.2)
        gone = [-(-int(v) // P) for v in model.lengths[done]]
        head = int(model.free_head)
        model.retire(done)
        taken += sum(gone)
        assert int(model.free_head) == head - sum(gone) and (model.lengths[done] == 0).all() and (model.block_table[done] == -1).all()
        pages_are_whole(model)
        for b in range(3):
            if done[b]:
                alone[b] = build(n_requests=1)
    assert taken > 3 * POOL and refused > 3
    model.retire(torch.ones(3, dtype=torch.bool))
    assert model.free_head.tolist() == [0] and model.lengths.tolist() == [0, 0, 0]
    pages_are_whole(model)


def test_retire_leaves_the_tables_of_the_last_step_and_checks_its_argument(monkeypatch):
    Library(monkeypatch)
    model = build()
    _, tables = model.step(tokens(9, 0), i32([4, 5, 0]))
    model.retire(torch.tensor([True, False, True]))
    assert tables.seq_len.tolist() == [4, 5, 0] and tables.free_head.tolist() == [3] and model.lengths.tolist() == [0, 5, 0] and model.free_head.tolist() == [2]
    for bad in (torch.tensor([1, 0, 1]), torch.tensor([True, False])):
        with pytest.raises((TypeError, ValueError), match="seats"):
            model.retire(bad)
    model.retire(torch.zeros(3, dtype=torch.bool))
    assert model.lengths.tolist() == [0, 5, 0] and model.free_head.tolist() == [2]
    _, tables = model.step(tokens(5, 1), i32([4, 1, 0]))
    assert tables.seq_len.tolist() == [4, 6, 0] and tables.request.tolist() == [0, 0, 0, 0, 1]
    pages_are_whole(model)
