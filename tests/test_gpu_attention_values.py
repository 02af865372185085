"""Attention, norm and rotation on the GPU where single values decide: weights with all of their bits, infinite values."""
import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from test_gpu_attention import DT, HALF_STEP, Cache, f64, i32, queries, rope_case
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


# ---------------------------------------------------------------------------- infinite values

def compare_infinite(c, kv, q, seq, dtype, places, window=0, table_row=None):
    """places: (request, token, element, value) put into V in every key/value head.  Elements where a row sees none of them keep their bits; where it does, they are what the
    definition gives: the infinity that it sees, or no number where it sees both."""
    P, dev = c.P, (c.table.cuda(), c.k.cuda())
    rows = None if table_row is None else i32(table_row)
    clean, lse = M.moe_attn_decode(kv, q.cuda(), i32(seq), *dev, c.v.cuda(), window=window, table_row=rows, want_lse=True)
    v = c.v.clone()
    for b, t, d, value in places:
        v[c.table[b, t // P].long(), :, t % P, d] = value
    out, lse2 = M.moe_attn_decode(kv, q.cuda(), i32(seq), *dev, v.cuda(), window=window, table_row=rows, want_lse=True)
    torch.cuda.synchronize()
    want = clean.float().cpu()
    assert want.isfinite().all() and torch.equal(lse, lse2)
    for r, n in enumerate(seq):
        request = r if table_row is None else table_row[r]
        first = max(0, n - window) if window else 0
        for d in {d for _, _, d, _ in places}:
            seen = [x for b, t, e, x in places if b == request and e == d and first <= t < n]
            if seen:
                want[r, :, d] = sum(seen)
    got = out.float().cpu()
    same = (got == want) | (got.isnan() & want.isnan())
    assert same.all(), (got[~same][:8], want[~same][:8], torch.nonzero(~same)[:8])


INF = float("inf")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [32, 64, 96, 128, 160, 192, 224, 256])
def test_attention_gives_the_infinity_of_a_value(D, dtype):
    lens = [1, 1, 2, 17, 33, 64, 300]
    c = Cache(lens, 2, D, 16, dtype, D)
    kv = M.make_kv_shape(6, 2, D, 16, c.table.shape[1], c.k.shape[0], dtype)
    q = queries(len(lens), kv, dtype, D + 1, std=0.5)
    places = [(0, 0, 3, INF), (1, 0, D - 1, -INF), (2, 1, 0, INF), (2, 0, 5, -INF), (3, 16, 7, INF), (4, 0, 9, -INF), (4, 32, 9, -INF), (5, 40, 11, INF), (5, 3, 11, -INF),
              (6, 299, 1, INF), (6, 0, 2, -INF), (6, 150, 4, INF), (6, 151, 4, INF)]
    for window in (0, 20):
        compare_infinite(c, kv, q, lens, dtype, places, window)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("scores", ["equal", "powers"])
def test_attention_gives_the_infinity_of_a_value_whatever_its_weight(dtype, scores):
    # every token of a request once: weights of exactly 1, and of about 2^-j down to the least that an exponential has
    n, D = 124, 64
    c = Cache([n] * n, 1, D, 16, dtype, 5)
    c.k = torch.zeros_like(c.k)
    if scores == "powers":
        t = torch.arange(n)
        for b in range(n):
            c.k[c.table[b, t // 16].long(), 0, t % 16, 0] = -t.to(c.k.dtype)
    kv = M.make_kv_shape(3, 1, D, 16, c.table.shape[1], c.k.shape[0], dtype)
    q = torch.zeros((n, 3, D), dtype=DT[dtype])
    q[..., 0] = 0.69140625                       # just below ln 2: token t weighs about 2^-t
    seq = [n] * n
    v = c.v.clone()
    for b in range(n):
        v[c.table[b, b // 16].long(), :, b % 16, 7] = INF
    for rows in (None, i32(list(range(n)))):
        out, _ = M.moe_attn_decode(kv, q.cuda(), i32(seq), c.table.cuda(), c.k.cuda(), v.cuda(), scale=1.0, table_row=rows)
        torch.cuda.synchronize()
        assert (out[:, :, 7] == INF).all(), (out[:, 0, 7] != INF).nonzero().flatten().tolist()
        others = torch.ones(D, dtype=torch.bool)
        others[7] = False
        assert out[:, :, others].isfinite().all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_q,n_kv", [(1, 1), (4, 1), (16, 2), (32, 8), (9, 1), (24, 1)])
def test_attention_gives_the_infinity_of_a_value_in_prompts(n_q, n_kv, dtype):
    lens = [37, 90, 3]
    c = Cache(lens, n_kv, 64, 16, dtype, n_q)
    kv = M.make_kv_shape(n_q, n_kv, 64, 16, c.table.shape[1], c.k.shape[0], dtype)
    rows = [0] * 37 + [-1] + [1] * 90 + [2] * 3
    seq = list(range(1, 38)) + [0] + list(range(1, 91)) + [1, 2, 3]
    q = queries(len(rows), kv, dtype, n_q + 1, std=0.5)
    places = [(0, 0, 3, INF), (0, 20, 8, -INF), (0, 33, 8, INF), (1, 64, 5, INF), (1, 40, 5, INF), (1, 89, 6, -INF), (1, 0, 7, -INF), (2, 2, 1, INF)]
    for window in (0, 11):
        compare_infinite(c, kv, q, seq, dtype, places, window, rows)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_gives_the_infinity_of_a_value_over_many_blocks(dtype):
    lens = [9000, 2500, 40]
    c = Cache(lens, 2, 128, 16, dtype, 3)
    kv = M.make_kv_shape(8, 2, 128, 16, c.table.shape[1], c.k.shape[0], dtype)
    q = queries(3, kv, dtype, 4, std=0.5)
    compare_infinite(c, kv, q, lens, dtype, [(0, 0, 1, INF), (0, 8999, 2, -INF), (0, 4000, 3, INF), (0, 7000, 3, -INF), (1, 1200, 100, INF), (1, 1201, 101, -INF), (2, 39, 9, INF)])


# ---------------------------------------------------------------------------- norm and rotation

@pytest.mark.parametrize("pairs", [False, True])
@pytest.mark.parametrize("T", [6, 600])          # eight wavefronts to a row, and four
@pytest.mark.parametrize("D,rot", [(64, 32), (128, 64), (96, 8), (64, 0), (256, 248)])
@pytest.mark.parametrize("x_dtype,dtype", [("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
def test_norm_rope_leaves_elements_behind_rot_dim_to_themselves(D, rot, T, pairs, x_dtype, dtype):
    kv, x, freq, pos, slots, _, caches = rope_case(T, 4, 2, D, 4, x_dtype, dtype, rot, pairs, False, D + rot)
    bad = [(1, 0, rot + 3, INF), (1, 0, rot + 4, -0.0), (2, 1, D - 1, -INF), (3, 3, rot, float("nan")), (0, 4, rot + 2, -INF), (T - 1, 5, rot + 5, INF), (T - 1, 2, rot + 1, INF), (T - 1, 2, rot + 6, -INF)]
    for t, h, d, value in bad:
        x[t, h * D + d] = value
    dev = [c.cuda() for c in caches]
    q = M.moe_qk_norm_rope(kv, x.cuda(), freq.cuda(), pos.cuda(), slots.cuda(), *dev, pairs=pairs)
    torch.cuda.synchronize()
    s = slots.long()
    k = dev[0].cpu()[s // 4, :, s % 4]
    heads = x.view(T, 8, D)[..., rot:].to(DT[dtype])
    for got, want in ((q.cpu()[..., rot:], heads[:, :4]), (k[..., rot:], heads[:, 4:6])):
        nan = want.isnan()
        assert torch.equal(got.isnan(), nan) and torch.equal(got[~nan], want[~nan]) and torch.equal(torch.signbit(got[~nan]), torch.signbit(want[~nan]))
    if rot:
        assert q[..., :rot].isfinite().all() and k[..., :rot].isfinite().all()
