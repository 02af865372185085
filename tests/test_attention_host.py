"""Attention over a paged cache without a GPU: shapes and arguments that the library refuses before anything is
enqueued, sizes of workspaces, and the oracle's tables against their definition."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import attention
from paper_2411_11217_amd import binding as B

FAKE = ctypes.c_void_p(1 << 12)                  # never dereferenced: the checks come first


def far(i):
    """Addresses that are 1 GiB apart, for arguments that must not overlap."""
    return ctypes.c_void_p((i + 1) << 30)


@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(n_q=8), 0), (dict(n_q=1024, n_kv=1), 0), (dict(head_dim=32), 0), (dict(head_dim=256), 0), (dict(page_tokens=1), 0), (dict(page_tokens=7), 0),
    (dict(n_kv=0), B.ERR_INVALID_ARG), (dict(n_q=0), B.ERR_INVALID_ARG), (dict(n_q=30), B.ERR_INVALID_ARG), (dict(n_q=1032), B.ERR_INVALID_ARG),
    (dict(n_q=4), B.ERR_INVALID_ARG), (dict(head_dim=0), B.ERR_INVALID_ARG), (dict(head_dim=80), B.ERR_INVALID_ARG), (dict(head_dim=288), B.ERR_INVALID_ARG),
    (dict(page_tokens=0), B.ERR_INVALID_ARG), (dict(max_pages=0), B.ERR_INVALID_ARG), (dict(pool_pages=0), B.ERR_INVALID_ARG), (dict(pool_pages=-1), B.ERR_INVALID_ARG),
    (dict(pool_pages=1 << 40), B.ERR_INVALID_ARG), (dict(pool_pages=1 << 27), B.ERR_INVALID_ARG), (dict(pool_pages=1 << 26), B.ERR_INVALID_ARG),
    (dict(pool_pages=(1 << 25) - 1), 0), (dict(max_pages=1 << 27), B.ERR_INVALID_ARG), (dict(dtype=2), B.ERR_UNSUPPORTED_DTYPE),
])
def test_kv_shapes(kw, code):
    base = dict(n_q=32, n_kv=8, head_dim=128, page_tokens=16, max_pages=64, dtype=1, pool_pages=1000)
    base.update(kw)
    assert M.kv_validate(B.KvShape(*[base[n] for n in ("n_q", "n_kv", "head_dim", "page_tokens", "max_pages", "dtype", "pool_pages")])) == code
    assert B._lib().moe_kv_validate(None) == B.ERR_INVALID_ARG


def kv(**kw):
    return M.make_kv_shape(**{**dict(n_q=8, n_kv=2, head_dim=64, page_tokens=16, max_pages=8, pool_pages=100, dtype="bf16"), **kw})


def test_assign_refusals():
    lib, s = B._lib(), kv()

    def call(B_=4, T=9, n_free=5, **kw):
        names = ["cached", "fresh", "free_pages", "free_head", "block_table", "seq_len", "row_start", "positions", "slots", "request", "free_head_out"]
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        return lib.moe_kv_assign(ctypes.byref(s), B_, T, p["cached"], p["fresh"], p["free_pages"], n_free, p["free_head"], p["block_table"], p["seq_len"], p["row_start"],
                                 p["positions"], p["slots"], p["request"], p["free_head_out"], None, None)

    assert call(B_=-1) == call(T=-1) == call(n_free=-1) == call(B_=4097) == call(T=1 << 30) == B.ERR_INVALID_ARG
    for name in ("cached", "fresh", "free_pages", "free_head", "block_table", "seq_len", "row_start", "positions", "slots", "request", "free_head_out"):
        assert call(**{name: None}) == B.ERR_INVALID_ARG, name
    # what is written must not be what is read
    assert call(seq_len=far(0)) == call(free_head_out=far(3)) == call(seq_len=ctypes.c_void_p((1 << 30) + 12)) == call(block_table=far(2)) == B.ERR_INVALID_ARG
    assert call(B_=0, T=0, **{n: None for n in ("cached", "fresh", "free_pages", "free_head")}) == 0            # nothing to do
    assert lib.moe_kv_assign(None, *[0] * 2, *[None] * 3, 0, *[None] * 10) == B.ERR_INVALID_ARG


def test_norm_rope_refusals():
    lib, s = B._lib(), kv()

    def call(T=3, dtype=0, row=768, eps=1e-5, rot=64, shape=s, **kw):
        names = ["qkv", "q_gamma", "k_gamma", "inv_freq", "positions", "slots", "q", "k_cache", "v_cache"]
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        return lib.moe_qk_norm_rope(ctypes.byref(shape), T, p["qkv"], dtype, row, p["q_gamma"], p["k_gamma"], eps, p["inv_freq"], rot, 0, p["positions"], p["slots"], p["q"],
                                    p["k_cache"], p["v_cache"], None, None)

    assert call(dtype=2) == B.ERR_UNSUPPORTED_DTYPE
    assert call(T=-1) == call(row=767) == call(row=764) == call(row=770) == call(dtype=1, row=772) == call(row=1 << 31) == B.ERR_INVALID_ARG
    assert call(rot=-8) == call(rot=72) == call(rot=4) == call(eps=-1.0) == call(eps=float("nan")) == B.ERR_INVALID_ARG
    for name in ("qkv", "inv_freq", "positions", "slots", "q", "k_cache", "v_cache"):
        assert call(**{name: None}) == B.ERR_INVALID_ARG, name
    for name in ("qkv", "q_gamma", "k_gamma", "q", "k_cache", "v_cache"):
        assert call(**{name: ctypes.c_void_p((20 << 30) + 8)}) == B.ERR_INVALID_ARG, name                       # alignment
    assert call(q=far(0)) == call(k_cache=far(8)) == call(k_cache=far(0)) == call(q=far(7)) == B.ERR_INVALID_ARG
    assert call(T=0, qkv=None) == 0


def test_attention_refusals_and_workspace():
    lib, s = B._lib(), kv()
    need = M.attn_workspace_bytes(s, 5)
    assert need >= 16384

    def call(R=5, table_rows=5, window=0, scale=0.1, ws=need, shape=s, **kw):
        names = ["q", "seq_len", "table_row", "block_table", "k_cache", "v_cache", "out", "lse", "workspace"]
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        return lib.moe_attn_decode(ctypes.byref(shape), R, p["q"], p["seq_len"], p["table_row"], p["block_table"], table_rows, p["k_cache"], p["v_cache"], window, scale,
                                   p["out"], p["lse"], p["workspace"], ws, None, None)

    assert call(ws=need - 1) == B.ERR_WORKSPACE_TOO_SMALL
    assert call(R=-1) == call(window=-1) == call(table_rows=0) == call(scale=float("nan")) == call(table_rows=4, table_row=None) == B.ERR_INVALID_ARG
    for name in ("q", "seq_len", "block_table", "k_cache", "v_cache", "out", "workspace"):
        assert call(**{name: None}) == B.ERR_INVALID_ARG, name
    for name in ("q", "k_cache", "v_cache", "out"):
        assert call(**{name: ctypes.c_void_p((20 << 30) + 8)}) == B.ERR_INVALID_ARG, name
    assert call(workspace=ctypes.c_void_p((20 << 30) + 128)) == B.ERR_INVALID_ARG
    assert call(out=far(0)) == call(out=far(4)) == call(out=far(5)) == call(lse=far(6)) == call(lse=far(0)) == B.ERR_INVALID_ARG       # written over what is read
    assert call(R=0, q=None) == 0
    assert lib.moe_attn_workspace_bytes(ctypes.byref(s), 5, None) == B.ERR_INVALID_ARG
    wide = kv(max_pages=(1 << 27) - 1)
    assert lib.moe_attn_workspace_bytes(ctypes.byref(wide), 17, ctypes.byref(ctypes.c_size_t())) == B.ERR_INVALID_ARG        # 17 * 2^27 tiles
    assert lib.moe_attn_workspace_bytes(ctypes.byref(wide), 9, ctypes.byref(ctypes.c_size_t())) == B.ERR_INVALID_ARG         # 9 rows of 2^27 - 1 tiles
    assert lib.moe_attn_workspace_bytes(ctypes.byref(wide), 8, ctypes.byref(ctypes.c_size_t())) == 0
    assert lib.moe_attn_workspace_bytes(ctypes.byref(kv(dtype="bf16", head_dim=256, n_q=1024, n_kv=1)), 100000, ctypes.byref(ctypes.c_size_t())) == 0


def test_binding_checks_before_the_library():
    s = kv()
    x = torch.zeros((3, 768))
    with pytest.raises(ValueError, match="qkv"):
        M.moe_qk_norm_rope(s, x, torch.zeros(32, dtype=torch.float64), None, None, None, None)                 # not on the device
    with pytest.raises(TypeError, match="qkv"):
        M.moe_qk_norm_rope(s, x.half(), torch.zeros(32, dtype=torch.float64), None, None, None, None)
    with pytest.raises(ValueError, match="step"):
        M.moe_kv_assign(s, torch.zeros(3, dtype=torch.int32), None, None, None, None)
    with pytest.raises(ValueError, match="q"):
        M.moe_attn_decode(s, torch.zeros((2, 8, 64), dtype=torch.bfloat16), None, None, None, None)
    assert M.make_kv_shape(8, 2, 64, 16, 8, 100, "f32").cache_shape == (100, 2, 16, 64)
    # what the calls read is that of the fields, also after one is set
    s = M.make_kv_shape(8, 2, 64, 16, 8, 100, "f32")
    assert s.known()[1:] == (torch.float32, (100, 2, 16, 64), 8, 64) and s.known()[0] is s.known()[0]
    s.head_dim, s.dtype = 128, 1
    assert s.known()[1:] == (torch.bfloat16, (100, 2, 16, 128), 8, 128)


def test_oracle_tables_by_hand():
    # three requests, pages of 4: 3 tokens + 2 (one new page), 4 + 1 (one new page), 0 + 9 (three, and only two are left)
    table = np.array([[7, -1, -1], [5, -1, -1], [-1, -1, -1]], np.int32)
    r = attention.assign(4, 3, 20, 14, [3, 4, 0], [2, 1, 9], [0, 11, 12, 13, 14], 1, table)
    assert r["seq_len"].tolist() == [5, 5, 0] and r["row_start"].tolist() == [0, 2, 3, 12] and r["free_head"].tolist() == [3] and r["status"] == 2
    assert r["block_table"].tolist() == [[7, 11, -1], [5, 12, -1], [-1, -1, -1]]
    assert r["positions"].tolist() == [3, 4, 4, 0, 1, 2, 3, 4, 5, 6, 7, 8, 0, 0]
    assert r["slots"].tolist() == [31, 44, 48] + [-1] * 11
    assert r["request"].tolist() == [0, 0, 1] + [2] * 9 + [-1] * 2


def test_oracle_attention_is_a_softmax():
    g = np.random.default_rng(0)
    q, k, v = g.normal(size=(3, 32)), g.normal(size=(5, 32)), g.normal(size=(5, 32))
    out, lse, bound, _ = attention.attend(q, k, v, 0.2, False)
    e = np.exp(0.2 * q @ k.T)
    assert np.allclose(out, e @ v / e.sum(-1, keepdims=True)) and np.allclose(lse, np.log(e.sum(-1))) and (bound > 0).all()
    out, lse, _, _ = attention.attend(q, k[:0], v[:0], 0.2, False)
    assert (out == 0).all() and (lse == -np.inf).all()
    y, _ = attention.qk_norm_rope(q[:, None], None, 0.0, [0.5, 0.25], [0, 1, 2], True)
    z = (q[:, 0] + 1j * q[:, 1]) * np.exp(0.5j * np.arange(3))
    assert np.allclose(y[:, 0, 0], z.real) and np.allclose(y[:, 0, 1], z.imag) and np.allclose(y[:, 0, 4:], q[:, 4:])


def test_tiles_are_dealt_to_blocks_once(tmp_path):
    """Random rows through the split's arithmetic, and the division by multiplication, under the host sanitizers."""
    import os
    import shutil
    import subprocess
    if not shutil.which("g++"):
        pytest.skip("no host compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    exe = str(tmp_path / "attn_split_driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I", os.path.join(root, "include"),
                        "-I", os.path.join(root, "paper_2411_11217_amd", "csrc"), os.path.join(root, "tests", "attn_split_driver.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
