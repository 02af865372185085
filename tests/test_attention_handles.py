"""Handles of the attention's calls on the host: shapes of a cache and tables of a step that are copied, pickled or changed stay their
own, and what reaches the library is what the handle of the call says."""
import copy
import ctypes
import pickle
import types

import pytest
import torch

import paper_2411_11217_amd as M
from paper_2411_11217_amd import binding as B

FIELDS = [n for n, _ in B.KvShape._fields_]


def values(kv):
    return [getattr(kv, n) for n in FIELDS]


def told(kv):
    """What a call tells the library: the structure behind the reference, and what the binding checks tensors against."""
    ref, dtype, cache_shape, n_q, head_dim = kv.known()
    assert (dtype, cache_shape, n_q, head_dim) == (kv.torch_dtype, kv.cache_shape, kv.n_q, kv.head_dim)
    return values(ctypes.cast(ref, ctypes.POINTER(B.KvShape)).contents)


@pytest.mark.parametrize("used", [False, True])
@pytest.mark.parametrize("how", [copy.copy, copy.deepcopy, lambda s: pickle.loads(pickle.dumps(s)), lambda s: B.KvShape.from_buffer_copy(s), lambda s: copy.copy(copy.deepcopy(s))])
def test_a_copied_shape_is_its_own(how, used):
    s = M.make_kv_shape(8, 2, 64, 16, 8, 100, "bf16")
    if used:
        s.known()
    c = how(s)
    assert type(c) is B.KvShape and values(c) == values(s)
    s.pool_pages, s.max_pages, s.head_dim = 1000000, 3, 128
    assert told(c) == [8, 2, 64, 16, 8, 1, 100] and told(s) == [8, 2, 128, 16, 3, 1, 1000000]
    c.dtype, c.page_tokens = 0, 5
    assert told(c) == [8, 2, 64, 5, 8, 0, 100] and told(s) == [8, 2, 128, 16, 3, 1, 1000000]
    d = how(c)                                   # and after both have been used
    c.n_q = 4
    assert told(d) == [8, 2, 64, 5, 8, 0, 100] and told(c) == [4, 2, 64, 5, 8, 0, 100]


def test_a_shape_changed_through_other_memory_is_read_again():
    s = M.make_kv_shape(8, 2, 64, 16, 8, 100, "bf16")
    assert s.known()[0] is s.known()[0]
    same = B.KvShape.from_buffer(s)
    s.known()
    same.pool_pages, same.dtype = 7, 0
    assert told(s) == [8, 2, 64, 16, 8, 0, 7] and told(same) == told(s)
    ctypes.pointer(s).contents.head_dim = 32
    assert told(s)[2] == 32 and told(same)[2] == 32


# ---------------------------------------------------------------------------- tables of a step

OUTPUTS = ("seq_len", "row_start", "positions", "slots", "request", "free_head")


class Recorder:
    """In place of the library: keeps the arguments of moe_kv_assign."""

    def __init__(self, monkeypatch):
        self.calls = []
        monkeypatch.setattr(B, "_lib", lambda: self)
        monkeypatch.setattr(B, "_dev", lambda t, dtype, shape, name: None if t is None else t.data_ptr())
        monkeypatch.setattr(B, "_stream", lambda stream: 0)

    def moe_kv_assign(self, *args):
        self.calls.append(args)
        return 0


@pytest.mark.parametrize("used", [False, True])
@pytest.mark.parametrize("how", [copy.deepcopy, lambda s: pickle.loads(pickle.dumps(s)), copy.copy, lambda s: s])
def test_a_copied_step_is_written_where_it_is_read(how, used, monkeypatch):
    lib = Recorder(monkeypatch)
    kv = M.make_kv_shape(1, 1, 32, 16, 8, 100, "bf16")
    args = [torch.zeros(n, dtype=torch.int32) for n in ((3,), (3,), (100,), (1,), (3, 8))]
    step = B.KvStep(kv, 3, 40, "cpu")
    if used:
        B.moe_kv_assign(kv, *args, step=step)
    other = how(step)
    assert B.moe_kv_assign(kv, *args, step=other) is other
    assert list(lib.calls[-1][9:15]) == [getattr(other, name).data_ptr() for name in OUTPUTS]
    assert lib.calls[-1][1:3] == (3, 40) and [getattr(other, name).numel() for name in OUTPUTS] == [3, 4, 40, 40, 40, 1]
    B.moe_kv_assign(kv, *args, step=step)
    assert list(lib.calls[-1][9:15]) == [getattr(step, name).data_ptr() for name in OUTPUTS]


# ---------------------------------------------------------------------------- streams

def test_the_current_device_is_asked_for_by_its_public_name(monkeypatch):
    # torch.cuda.current_device initialises the device, and refuses in a child that was forked from a process that has
    asked = []
    monkeypatch.setattr(torch.cuda, "current_device", lambda: asked.append("device") or 3)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda device: 1000 + device, raising=False)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: 5, raising=False)
    assert B._stream(None) == 1003 and asked == ["device"]
    assert B._stream(77) == 77


# ---------------------------------------------------------------------------- whole numbers

@pytest.mark.parametrize("window,told_window", [(0, 0), (5, 5), (2 ** 31 - 1, 2 ** 31 - 1), (2 ** 31, 2 ** 31 - 1), (2 ** 32, 2 ** 31 - 1), (2 ** 32 + 5, 2 ** 31 - 1),
                                                (2 ** 63 - 1, 2 ** 31 - 1), (-1, -1), (-2 ** 32, -1), (-2 ** 33 + 1, -1)])
def test_a_window_beyond_32_bits_is_not_cut_to_its_low_bits(window, told_window, monkeypatch):
    # longer than any row is all of it, and what is negative stays refused
    lib = Recorder(monkeypatch)
    lib.moe_attn_decode = lambda *args: lib.calls.append(args) or 0
    kv = M.make_kv_shape(2, 1, 32, 16, 8, 100, "bf16")
    q, cache = torch.zeros((3, 2, 32), dtype=torch.bfloat16), torch.zeros(kv.cache_shape, dtype=torch.bfloat16)
    workspace = types.SimpleNamespace(buf=torch.zeros(16))
    B.moe_attn_decode(kv, q, torch.zeros(3, dtype=torch.int32), torch.zeros((3, 8), dtype=torch.int32), cache, cache, window=window, out=q.clone(), workspace=workspace)
    assert ctypes.c_int32(lib.calls[-1][9]).value == told_window
