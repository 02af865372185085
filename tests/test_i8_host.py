"""The layer in 8-bit integers on the host: shapes, page geometry and packing, what the entry points refuse before anything is enqueued, the oracle's own
values, and what DecodeLayers takes.  No kernel is launched here."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import int8 as O
from paper_2411_11217_amd import binding as B


def far(i, off=0):
    """A pointer of its own gigabytes: never followed, the calls here are refused or do nothing."""
    return ctypes.c_void_p(((20 + 20 * i) << 30) + off)


def shape(T=3, H=256, F=512, E=4, k=2, dtype="i8", page=65536):
    return M.make_shape(T, H, F, E, k, dtype, page)


# ---------------------------------------------------------------------------- shapes and pages

@pytest.mark.parametrize("kw,code", [
    (dict(), 0), (dict(T=0), 0), (dict(H=130816, F=256), 0), (dict(H=256, F=130816), 0),
    (dict(H=384), B.ERR_INVALID_ARG), (dict(F=128), B.ERR_INVALID_ARG), (dict(H=131072), B.ERR_INVALID_ARG), (dict(F=131072), B.ERR_INVALID_ARG),
    (dict(page=8192), B.ERR_INVALID_ARG), (dict(page=16384), 0), (dict(k=5), B.ERR_INVALID_ARG), (dict(T=-1), B.ERR_INVALID_ARG),
])
def test_shapes(kw, code):
    assert M.validate_shape(shape(**kw)) == code


def test_page_geometry():
    s = shape(H=4096, F=14336, E=8, page=2 << 20)
    assert M.tile_bytes(s) == 16384 and M.pages_required(s) == (56, 28)          # half of bf16's
    assert M.linear_pages_required(M.make_linear_shape(1, 4096, 6144, 65536, "i8")) == 384
    for K, N in ((128, 128), (384, 128), (131072, 128), (256, 64)):
        with pytest.raises(M.MoEError):
            M.linear_pages_required(M.make_linear_shape(1, K, N, 65536, "i8"))


def test_pack_unpack_round_trip_and_layout():
    s = shape(H=512, F=768, E=3, page=3 * 16384)
    g = torch.Generator().manual_seed(2)
    W1, W3, W2 = (torch.randint(-128, 128, n, dtype=torch.int8, generator=g) for n in ((3, 768, 512), (3, 768, 512), (3, 512, 768)))
    pw = M.PagedWeights(s, W1, W3, W2, order=g, extra_pages=4)
    assert all(torch.equal(a, b) for a, b in zip(pw.unpack(), (W1, W3, W2)))
    # tile (f / 128, w, h / 128); inside it the 16-byte chunk c (0 .. 7) of row n in half c >> 2 at position (c & 3) ^ ((n >> 2) & 2)
    e, ft, w, kt, n = 1, 4, 1, 3, 77
    t = (ft * 2 + w) * (512 // 128) + kt
    page = pw.pages_host[int(pw.table_host[e, t // 3])].view(torch.int8)[(t % 3) * 16384:]
    for c in range(8):
        at = (c >> 2) * 8192 + n * 64 + (((c & 3) ^ ((n >> 2) & 2)) << 4)
        k = kt * 128 + c * 16
        assert torch.equal(page[at:at + 16], W3[e, ft * 128 + n, k:k + 16])
    ls = M.make_linear_shape(1, 768, 256, 5 * 16384, "i8")
    W = torch.randint(-128, 128, (256, 768), dtype=torch.int8, generator=g)
    pages = M.linear_pages_required(ls)
    out = torch.full((pages + 1, 5 * 16384), 7, dtype=torch.uint8)
    table = torch.tensor([2, 0, 3], dtype=torch.int32)
    assert pages == 3
    M.linear_pack(ls, W, table, out)
    t = 1 * 6 + 4                                # second column tile, fifth tile along k
    page = out[int(table[t // 5])].view(torch.int8)[(t % 5) * 16384:]
    c, n = 5, 9
    at = (c >> 2) * 8192 + n * 64 + (((c & 3) ^ ((n >> 2) & 2)) << 4)
    assert torch.equal(page[at:at + 16], W[128 + n, 4 * 128 + c * 16:4 * 128 + c * 16 + 16])
    assert (out[1] == 7).all() and (out[3][2 * 16384:] == 0).all()               # no page's slot, and the padding of the last page
    with pytest.raises(ValueError):
        M.linear_pack(ls, W.to(torch.bfloat16), table, out)
    with pytest.raises(ValueError):
        M.PagedWeights(s, W1.to(torch.bfloat16), W3, W2)


def test_the_other_calls_refuse_8_bit_shapes():
    lib, s, p = B._lib(), shape(), far(0)
    ref = ctypes.byref(s)
    assert lib.moe_route(ref, p, p, None, p, p, None, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_permute(ref, p, p, None, p, p, p, p, None, None, p, 1 << 30, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_expert_ffn(ref, p, p, p, p, 10, None, p, p, None, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_layer(ref, p, p, None, p, p, 10, p, p, 1 << 30, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_layer_static(ref, p, p, None, p, p, 10, p, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_workspace_layout_get(ref, ctypes.byref(B.WorkspaceLayout())) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_stream_create(ref, p, 10, p, p, p, ctypes.byref(ctypes.c_void_p())) == B.ERR_UNSUPPORTED_DTYPE
    n = ctypes.c_int64()
    assert lib.moe_pipeline_pool_pages(ref, 2, 1, ctypes.byref(n)) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_pipeline_create(ref, 2, 1, p, p, p, 1, p, 10, p, ctypes.byref(ctypes.c_void_p())) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_post_attention_workspace_bytes(ref, ctypes.byref(ctypes.c_size_t())) == B.ERR_UNSUPPORTED_DTYPE
    ls = ctypes.byref(M.make_linear_shape(3, 256, 128, 65536, "i8"))
    assert lib.moe_linear(ls, p, p, p, 10, p, p, 16, None, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_pre_attention(ls, p, p, p, 1e-5, p, p, 10, p, p, p, None, p, 16, None) == B.ERR_UNSUPPORTED_DTYPE
    bf16 = M.make_linear_shape(3, 256, 256, 65536)
    assert lib.moe_post_attention(ref, ctypes.byref(bf16), p, p, p, p, 1e-5, p, None, p, p, 10, p, p, p, p, 1 << 30, None) == B.ERR_UNSUPPORTED_DTYPE
    # and the calls for 8-bit integers all others
    f = ctypes.byref(shape(dtype="bf16"))
    size = ctypes.c_size_t()
    assert lib.moe_layer_i8_workspace_bytes(f, ctypes.byref(size)) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_linear_i8(ctypes.byref(bf16), p, p, p, p, 10, p, p, None, None) == B.ERR_UNSUPPORTED_DTYPE
    assert lib.moe_post_attention_i8_workspace_bytes(ref, ctypes.byref(bf16), ctypes.byref(size)) == B.ERR_UNSUPPORTED_DTYPE
    assert s.routed().dtype == M.DTYPE_BF16 and M.validate_shape(s.routed()) == 0 and shape(dtype="f32").routed().dtype == M.DTYPE_F32


# ---------------------------------------------------------------------------- refusals

def test_quantize_refusals():
    lib = B._lib()

    def call(T=3, N=64, dtype=1, row=64, x=far(0), q=far(1), scale=far(2)):
        return lib.moe_quantize_i8(T, N, x, dtype, row, q, scale, None)

    assert call(dtype=2) == call(dtype=-1) == B.ERR_UNSUPPORTED_DTYPE
    assert call(T=-1) == call(N=0) == call(N=62, row=64) == call(row=60) == call(row=66) == call(row=1 << 31) == B.ERR_INVALID_ARG
    assert call(x=None) == call(q=None) == call(scale=None) == B.ERR_INVALID_ARG
    assert call(x=far(0, 4)) == call(x=far(0, 8), dtype=0) == call(q=far(1, 2)) == call(scale=far(2, 2)) == B.ERR_INVALID_ARG
    assert call(q=far(0, 128)) == call(scale=far(0, 3 * 128 - 4)) == call(scale=far(1, 100)) == B.ERR_INVALID_ARG            # written over what is read
    assert call(T=0, x=None, q=None, scale=None) == 0


def test_norm_refusals():
    lib = B._lib()
    names = ["hidden", "delta", "gamma", "hidden_out", "x_out", "x_q", "x_scale"]

    def call(T=3, H=256, eps=1e-5, **kw):
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        return lib.moe_add_rmsnorm_i8(T, H, p["hidden"], p["delta"], p["gamma"], eps, p["hidden_out"], p["x_out"], p["x_q"], p["x_scale"], None)

    assert call(T=-1) == call(H=0) == call(H=254) == call(H=8196) == call(eps=-1.0) == call(eps=float("nan")) == B.ERR_INVALID_ARG
    for n in ("delta", "gamma", "x_q", "x_scale"):
        assert call(**{n: None}) == B.ERR_INVALID_ARG, n
    for i, n in enumerate(names[:4]):
        assert call(**{n: far(i, 8)}) == B.ERR_INVALID_ARG, n
    assert call(x_out=far(4, 4)) == call(x_q=far(5, 2)) == call(x_scale=far(6, 2)) == B.ERR_INVALID_ARG
    for out in names[3:]:                        # nothing is written over what is read, but the residual stream in place
        for i, other in enumerate(names):
            same = out == "hidden_out" and other in ("hidden", "delta")
            if other != out and not same:
                assert call(**{out: far(i)}) == B.ERR_INVALID_ARG, (out, other)
    assert call(hidden_out=far(0, 16)) == call(hidden_out=far(1, 1024)) == B.ERR_INVALID_ARG
    assert call(T=0, delta=None) == 0


def test_linear_refusals():
    lib = B._lib()
    names = ["x_q", "x_scale", "table", "pool", "w_scale", "out"]

    def call(T=3, K=256, N=128, pages=10, **kw):
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        s = M.make_linear_shape(T, K, N, 65536, "i8")
        return lib.moe_linear_i8(ctypes.byref(s), p["x_q"], p["x_scale"], p["table"], p["pool"], pages, p["w_scale"], p["out"], None, None)

    assert call(K=128) == call(K=320) == call(N=192) == call(K=131072) == call(T=-1) == call(pages=0) == B.ERR_INVALID_ARG
    for n in names:
        assert call(**{n: None}) == B.ERR_INVALID_ARG, n
    assert call(x_q=far(0, 8)) == call(pool=far(3, 8)) == call(out=far(0)) == call(out=far(1)) == B.ERR_INVALID_ARG
    assert call(T=0, x_q=None) == 0
    assert lib.moe_linear_i8(None, *[None] * 4, 0, *[None] * 4) == B.ERR_INVALID_ARG


def scales(**kw):
    v = dict(w1=30, w3=31, w2=32)
    v.update(kw)
    return (ctypes.c_void_p * 3)(*[None if i is None else far(i).value for i in (v["w1"], v["w3"], v["w2"])])


def test_expert_refusals():
    lib = B._lib()
    names = ["x_q", "x_scale", "row_src", "offsets", "table", "pool", "h", "h_q", "h_scale", "out"]

    def call(s=None, pages=10, sc=None, **kw):
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        s = shape() if s is None else s
        return lib.moe_expert_ffn_i8(ctypes.byref(s), p["x_q"], p["x_scale"], p["row_src"], p["offsets"], p["table"], p["pool"], pages, scales() if sc is None else sc, None,
                                     p["h"], p["h_q"], p["h_scale"], p["out"], None, None)

    assert call(pages=0) == call(s=shape(H=384)) == call(s=shape(T=1 << 22, H=1024, k=1)) == B.ERR_INVALID_ARG
    for n in names:
        if n != "row_src":
            assert call(**{n: None}) == B.ERR_INVALID_ARG, n
    for i, n in ((0, "x_q"), (5, "pool"), (6, "h"), (7, "h_q"), (9, "out")):
        assert call(**{n: far(i, 8)}) == B.ERR_INVALID_ARG, n
    for n in ("w1", "w3", "w2"):
        assert call(sc=scales(**{n: None})) == B.ERR_INVALID_ARG, n
    for out in ("h", "h_q", "h_scale", "out"):
        for i, other in enumerate(names):
            if other in ("x_q", "x_scale", "h", "h_q", "h_scale", "out") and other != out:
                assert call(**{out: far(i)}) == B.ERR_INVALID_ARG, (out, other)
    assert lib.moe_expert_ffn_i8(ctypes.byref(shape(dtype="bf16")), *[far(0)] * 6, 10, scales(), *[far(0)] * 7) == B.ERR_UNSUPPORTED_DTYPE
    assert call(s=shape(T=0), x_q=None) == 0


def test_layer_and_task_refusals():
    lib, s = B._lib(), shape()
    need = M.layer_i8_workspace_bytes(s)
    names = ["x", "x_q", "x_scale", "Wr", "table", "pool", "y", "workspace"]

    def layer(s=s, ws=need, pages=10, sc=None, **kw):
        p = {n: far(i) for i, n in enumerate(names)}
        p.update(kw)
        return lib.moe_layer_i8(ctypes.byref(s), p["x"], p["x_q"], p["x_scale"], p["Wr"], None, p["table"], p["pool"], pages, scales() if sc is None else sc, p["y"], p["workspace"],
                                ws, None)

    assert layer(ws=need - 1) == B.ERR_WORKSPACE_TOO_SMALL
    for n in names:
        assert layer(**{n: None}) == B.ERR_INVALID_ARG, n
    assert layer(workspace=far(7, 128)) == layer(x_q=far(1, 8)) == layer(pages=0) == layer(sc=scales(w2=None)) == B.ERR_INVALID_ARG
    assert layer(s=shape(dtype="bf16")) == B.ERR_UNSUPPORTED_DTYPE and layer(s=shape(T=0), x=None) == 0

    pre_names = ["hidden", "delta", "gamma", "table", "pool", "scale", "hidden_out", "x_q", "x_scale", "qkv"]

    def pre(T=3, K=256, N=384, eps=1e-5, pages=10, dtype="i8", **kw):
        p = {n: far(i) for i, n in enumerate(pre_names)}
        p.update(kw)
        ls = M.make_linear_shape(T, K, N, 65536, dtype)
        return lib.moe_pre_attention_i8(ctypes.byref(ls), p["hidden"], p["delta"], p["gamma"], eps, p["table"], p["pool"], pages, p["scale"], p["hidden_out"], p["x_q"], p["x_scale"],
                                        p["qkv"], None, None)

    for n in pre_names[1:]:
        assert pre(**{n: None}) == B.ERR_INVALID_ARG, n
    assert pre(eps=-1.0) == pre(pages=0) == pre(K=8448) == pre(x_q=far(7, 4)) == pre(qkv=far(7)) == pre(qkv=far(6)) == pre(x_q=far(1)) == B.ERR_INVALID_ARG
    assert pre(dtype="bf16") == B.ERR_UNSUPPORTED_DTYPE and pre(T=0, delta=None) == 0

    o = M.make_linear_shape(3, 512, 256, 65536, "i8")
    size = M.binding.post_attention_i8_workspace_bytes(s, o)
    assert size > need
    post_names = ["attn", "hidden", "o_table", "o_scale", "gamma", "Wr", "table", "pool", "hidden_mid", "x_moe", "y", "workspace"]

    def post(s=s, o=o, eps=1e-5, ws=size, pages=10, sc=None, **kw):
        p = {n: far(i) for i, n in enumerate(post_names)}
        p.update(kw)
        return lib.moe_post_attention_i8(ctypes.byref(s), ctypes.byref(o), p["attn"], p["hidden"], p["o_table"], p["o_scale"], p["gamma"], eps, p["Wr"], None, p["table"], p["pool"], pages,
                                         scales() if sc is None else sc, p["hidden_mid"], p["x_moe"], p["y"], p["workspace"], ws, None)

    assert post(ws=size - 1) == B.ERR_WORKSPACE_TOO_SMALL
    for n in post_names:
        assert post(**{n: None}) == B.ERR_INVALID_ARG, n
    assert post(eps=float("nan")) == post(pages=0) == post(workspace=far(11, 64)) == post(attn=far(0, 4)) == post(x_moe=far(9, 8)) == B.ERR_INVALID_ARG
    assert post(o=M.make_linear_shape(4, 512, 256, 65536, "i8")) == post(o=M.make_linear_shape(3, 512, 512, 65536, "i8")) == B.ERR_INVALID_ARG
    assert post(o=M.make_linear_shape(3, 512, 256, 16384, "i8")) == B.ERR_INVALID_ARG
    assert post(o=M.make_linear_shape(3, 512, 256, 65536)) == post(s=shape(dtype="bf16")) == B.ERR_UNSUPPORTED_DTYPE
    z = shape(T=0)
    assert post(s=z, o=M.make_linear_shape(0, 512, 256, 65536, "i8"), attn=None) == 0


def test_binding_checks_before_the_library():
    """Host tensors, other types and shapes are refused by name."""
    x = torch.zeros((3, 64))
    with pytest.raises(ValueError, match="x: must be"):
        M.moe_quantize_i8(x)
    with pytest.raises(ValueError, match="two dimensions"):
        M.moe_quantize_i8(x[0])
    with pytest.raises(ValueError, match="delta"):
        M.moe_add_rmsnorm_i8(None, x, torch.ones(64), 1e-5)
    ls = M.make_linear_shape(3, 256, 128, 65536, "i8")
    with pytest.raises(ValueError, match="x_q"):
        M.moe_linear_i8(ls, torch.zeros((3, 256), dtype=torch.int8), torch.ones(3), torch.zeros(1, dtype=torch.int32), torch.zeros((1, 65536), dtype=torch.uint8), torch.ones(128))
    with pytest.raises(KeyError):
        M.make_linear_shape(3, 256, 128, 65536, "f32")


def test_tensors_of_another_device_are_refused(monkeypatch):
    class On:
        def __init__(self, device):
            self.get_device = lambda: device

    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    B._here(On(1), None, On(1))
    with pytest.raises(ValueError, match="device 0, the current device is 1"):
        B._here(On(1), None, On(0))


# ---------------------------------------------------------------------------- the oracle

def test_oracle_quantize():
    """Half steps go to the even number, a row's largest value to 127, tiny rows keep a scale of 2^-126, rows that are not finite are NaN."""
    v = np.array([[127.0, 0.5, 1.5, -0.5, -2.5, 126.5], [0, 0, 0, 0, 0, -0.0], [1e-40, -3e-39, 0, 0, 0, 2e-38], [1, np.inf, 0, 0, 0, 0], [1, 0, 0, np.nan, 0, 0], [-3e38, 3.4e38, 1e30, 0, 0, 0]],
                 dtype=np.float32)
    q, s = O.quantize(v)
    assert q[0].tolist() == [127, 0, 2, 0, -2, 126] and s[0] == 1.0
    assert (q[1] == 0).all() and s[1] == s[2] == np.float32(2.0 ** -126)
    assert np.abs(q[2] * s[2].astype(np.float64) - v[2]).max() <= 2.0 ** -127
    assert np.isnan(s[3:5]).all() and (q[3:5] == 0).all()
    assert q[5].tolist() == [-112, 127, 0, 0, 0, 0] and np.isfinite(s[5])
    rng = np.random.default_rng(0)
    v = (rng.standard_normal((50, 300)) * 10.0 ** rng.integers(-30, 30, (50, 1))).astype(np.float32)
    q, s = O.quantize(v)
    assert (np.abs(q * s[:, None].astype(np.float64) - v) <= s[:, None] * (0.5 + 127 * 4 * O.U)).all() and (np.abs(q).max(axis=1) == 127).all()


def test_oracle_product_is_exact_in_its_sums():
    rng = np.random.default_rng(1)
    x, W = rng.integers(-128, 128, (3, 2000)).astype(np.int8), rng.integers(-128, 128, (5, 2000)).astype(np.int8)
    one = np.ones(5, np.float32)
    assert (O.product(x, one[:3], W, one) == x.astype(np.int64) @ W.astype(np.int64).T).all()


# ---------------------------------------------------------------------------- DecodeLayers

def test_decode_layers_takes_scales_with_8_bit_weights_only():
    kv = M.make_kv_shape(4, 1, 64, 4, 6, 14, "bf16")
    freq = torch.zeros(16, dtype=torch.float64)
    plain = [M.LayerWeights(*[None] * 7)]
    scaled = [M.LayerWeights(*[None] * 7, scales=M.LayerScales(None, None, None))]
    M.DecodeLayers(shape(1), kv, scaled, freq, 2, device="cpu")
    M.DecodeLayers(shape(1, dtype="bf16"), kv, plain, freq, 2, device="cpu")
    for s, layers in ((shape(1), plain), (shape(1, dtype="bf16"), scaled), (shape(1, dtype="f32"), plain)):
        with pytest.raises(ValueError):
            M.DecodeLayers(s, kv, layers, freq, 2, device="cpu")
    with pytest.raises(M.MoEError):              # queries of 3 * 32: no multiple of 256
        M.DecodeLayers(shape(1), M.make_kv_shape(3, 1, 32, 4, 6, 14, "bf16"), scaled, freq, 2, device="cpu")
