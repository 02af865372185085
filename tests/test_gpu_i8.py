"""The layer in 8-bit integers on the GPU against plain numpy (oracle/int8.py): quantised rows exactly, products within the roundings of their float32
arithmetic, at sizes, strides, page orders and values where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2411_11217_amd as M
from oracle import int8 as O
from paper_2411_11217_amd import binding as B

pytestmark = pytest.mark.gpu
INF, NAN = float("inf"), float("nan")


def bf16_values(t):
    return t.float().numpy()


def rows_of(T, N, dtype, seed, std=1.3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((T, N), generator=g) * std
    x[:, 0] += torch.arange(T) % 3               # rows of different scale
    return x.to(torch.bfloat16) if dtype == "bf16" else x


def check_quantized(x, q, scale, what=""):
    want_q, want_scale = O.quantize(x.float().numpy())
    np.testing.assert_array_equal(scale.cpu().numpy().view(np.uint32) & 0x7fffffff, want_scale.view(np.uint32) & 0x7fffffff, err_msg=what)
    np.testing.assert_array_equal(q.cpu().numpy(), want_q, err_msg=what)


# ---------------------------------------------------------------------------- rows in 8 bits

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,N", [(1, 4), (1, 8), (3, 12), (5, 260), (36, 4096), (17, 1020), (4, 1024), (3, 1028), (2, 2052), (9, 2820), (3, 4100), (2, 8196), (2, 14336), (3, 16384), (2, 16388),
                                 (1, 40000), (1000, 64), (777, 516)])
def test_quantize(T, N, dtype):
    x = rows_of(T, N, dtype, T + N)
    q, scale = M.moe_quantize_i8(x.cuda())
    check_quantized(x, q, scale)


@pytest.mark.parametrize("dtype,N,wide,first", [("bf16", 2820, 2832, 0), ("bf16", 512, 1024, 4), ("f32", 512, 1024, 4), ("f32", 4100, 4104, 0), ("bf16", 4096, 6144, 2048), ("bf16", 16640, 16644, 4),
                                                ("bf16", 64, 8192, 12)])
def test_quantize_rows_of_a_wider_matrix(dtype, N, wide, first):
    x = rows_of(23, wide, dtype, N)
    q, scale = M.moe_quantize_i8(x.cuda()[:, first:first + N])
    check_quantized(x[:, first:first + N], q, scale)
    # and into the middle of a buffer, whose neighbours stay
    buf = torch.full((23 * N + 64,), 55, dtype=torch.int8, device="cuda")
    scales = torch.full((25,), 7.0, device="cuda")
    q, scale = M.moe_quantize_i8(x.cuda()[:, first:first + N], x_q=buf[32:32 + 23 * N].view(23, N), x_scale=scales[1:24])
    check_quantized(x[:, first:first + N], q, scale)
    assert (buf[:32] == 55).all() and (buf[-32:] == 55).all() and scales[0] == 7 and scales[24] == 7


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [8, 260, 4096, 20000])
def test_quantize_values(dtype, N):
    """Zeros, ties, the largest and smallest numbers, one value alone, infinities and NaN in first, last and middle places."""
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    big, tiny = float(torch.finfo(dt).max), 2.0 ** -126
    rows = [torch.zeros(N), torch.full((N,), -0.0), torch.full((N,), big), torch.full((N,), -big), torch.full((N,), tiny), torch.linspace(-1, 1, N) * 2.0 ** -120, torch.linspace(-1, 1, N) * 2.0 ** -130]
    ties = (torch.arange(N) % 253 - 126).float() + 0.5           # with the largest at 127: halves of a step
    ties[N // 2] = 127.0
    rows += [ties, -ties, ties * 2.0 ** -40]
    for at in (0, N // 3, N - 1):
        one = torch.zeros(N)
        one[at] = -3.25
        rows.append(one)
        for bad in (INF, -INF, NAN):
            r = torch.linspace(-2, 2, N)
            r[at] = bad
            rows.append(r)
    both = torch.linspace(-2, 2, N)
    both[1], both[N - 2] = INF, NAN
    x = torch.stack(rows + [both]).to(dt)
    q, scale = M.moe_quantize_i8(x.cuda())
    check_quantized(x, q, scale)


# ---------------------------------------------------------------------------- residual and norm with rows in 8 bits

def check_norm(hidden, delta, gamma, eps, got):
    s, y, rel = O.rmsnorm(None if hidden is None else hidden.numpy(), delta.numpy(), gamma.numpy(), eps)
    hs, x, q, scale = (None if t is None else t.cpu() for t in got)
    if hs is not None:
        np.testing.assert_array_equal(hs.numpy(), s)
    slack = np.abs(y) * rel + 1e-300
    if x is not None:
        assert (np.abs(x.double().numpy() - y) <= slack + (np.abs(y) + slack) * O.U16).all()
    most = np.abs(y).max(axis=1)
    step = scale.double().numpy()
    want = np.maximum(most / 127, 2.0 ** -126)
    assert (np.abs(step - want) <= want * (rel + 2 * O.U)).all()
    # the quotient is formed by a product with a rounded inverse: 127 * 3 U of a step beside the value's own error
    off = np.abs(q.numpy() * step[:, None] - y)
    assert (off <= step[:, None] * (0.5 + 127 * 4 * O.U) + slack + np.abs(y) * 2 * O.U).all()
    assert np.abs(q.numpy()).max(axis=1).min() == 127


@pytest.mark.parametrize("T,H", [(1, 4), (5, 256), (3, 260), (7, 1024), (2, 1028), (36, 4096), (4, 4100), (9, 6144), (3, 8188), (2, 8192), (700, 128)])
@pytest.mark.parametrize("first,want_hidden,want_x", [(False, True, True), (True, True, False), (False, False, True)])
def test_norm(T, H, first, want_hidden, want_x):
    g = torch.Generator().manual_seed(T * H)
    hidden = None if first else torch.randn((T, H), generator=g) * 3
    delta, gamma = torch.randn((T, H), generator=g), 1 + 0.2 * torch.randn(H, generator=g)
    gamma[H // 2] = -1.5
    got = M.moe_add_rmsnorm_i8(None if first else hidden.cuda(), delta.cuda(), gamma.cuda(), 1e-5, want_hidden=want_hidden, want_x=want_x)
    assert (got[0] is None) == (not want_hidden) and (got[1] is None) == (not want_x)
    check_norm(hidden, delta, gamma, 1e-5, got)


def test_norm_values():
    """Rows of zeros, of tiny and of huge values, a gamma of zero, an infinity and a NaN, which stay in their rows."""
    H = 512
    g = torch.Generator().manual_seed(1)
    delta, gamma = torch.randn((8, H), generator=g), torch.ones(H)
    gamma[3] = 0.0
    delta[1] = 0.0
    delta[2] *= 1e-18
    delta[3] *= 1e17
    delta[5, 7] = INF
    delta[6, H - 1] = NAN
    hs, x, q, scale = (t.cpu() for t in M.moe_add_rmsnorm_i8(None, delta.cuda(), gamma.cuda(), 1e-6))
    np.testing.assert_array_equal(hs.numpy().view(np.uint32)[[0, 1, 2, 3, 4, 5, 7]], delta.numpy().view(np.uint32)[[0, 1, 2, 3, 4, 5, 7]])
    assert torch.isnan(scale[[5, 6]]).all() and (q[[5, 6]] == 0).all()
    assert (q[1] == 0).all() and scale[1] == 2.0 ** -126 and (x[1] == 0).all()
    keep = [0, 2, 3, 4, 7]
    check_norm(None, delta[keep], gamma, 1e-6, (hs[keep], x[keep], q[keep], scale[keep]))


def test_norm_in_place_in_the_residual_stream():
    """hidden_out may be hidden or delta, through the C ABI."""
    T, H = 9, 1280
    g = torch.Generator().manual_seed(4)
    hidden, delta, gamma = torch.randn((T, H), generator=g), torch.randn((T, H), generator=g), torch.ones(H)
    for which in (0, 1):
        h, d, ga = hidden.cuda(), delta.cuda(), gamma.cuda()
        q, scale = torch.empty((T, H), dtype=torch.int8, device="cuda"), torch.empty(T, device="cuda")
        out = (h, d)[which]
        assert B._lib().moe_add_rmsnorm_i8(T, H, h.data_ptr(), d.data_ptr(), ga.data_ptr(), 1e-5, out.data_ptr(), None, q.data_ptr(), scale.data_ptr(), B._stream(None)) == 0
        check_norm(hidden, delta, gamma, 1e-5, (out, None, q, scale))


# ---------------------------------------------------------------------------- the linear map

class Linear:
    def __init__(self, K, N, page=16384, seed=0, extra=3):
        g = torch.Generator().manual_seed(seed + K + N)
        self.K, self.N, self.page = K, N, page
        self.W = torch.randint(-128, 128, (N, K), dtype=torch.int8, generator=g)
        self.w_scale = torch.rand(N, generator=g) * 1e-3 + 1e-4
        ls = M.make_linear_shape(1, K, N, page, "i8")
        n = M.linear_pages_required(ls)
        self.table = torch.randperm(n + extra, generator=g)[:n].to(torch.int32)
        host = torch.randint(0, 255, (n + extra, page), dtype=torch.uint8, generator=g)
        M.linear_pack(ls, self.W, self.table, host)
        self.pool, self.dev_table, self.dev_scale = host.cuda(), self.table.cuda(), self.w_scale.cuda()

    def rows(self, T, seed=1):
        g = torch.Generator().manual_seed(seed + T)
        return torch.randint(-128, 128, (T, self.K), dtype=torch.int8, generator=g), torch.rand(T, generator=g) * 0.05 + 0.001

    def run(self, q, scale, **kw):
        return M.moe_linear_i8(M.make_linear_shape(q.shape[0], self.K, self.N, self.page, "i8"), q.cuda(), scale.cuda(), self.dev_table, self.pool, self.dev_scale, **kw)

    def check(self, q, scale, out):
        want = O.product(q.numpy(), scale.numpy(), self.W.numpy(), self.w_scale.numpy())
        off = np.abs(out.cpu().numpy().astype(np.float64) - want)
        assert (off <= np.abs(want) * O.PRODUCT).all(), float((off / np.maximum(np.abs(want), 1e-30)).max())


@pytest.mark.parametrize("K,N,page", [(256, 128, 16384), (256, 384, 3 * 16384), (512, 1152, 65536), (1280, 640, 16384 * 7), (4096, 512, 2 << 20), (2304, 2944, 65536), (768, 8192, 65536),
                                      (256, 20480, 65536), (10752, 256, 65536)])
def test_linear(K, N, page):
    lin = Linear(K, N, page)
    for T in (1, 2, 15, 16, 17, 33, 64, 65, 100, 128, 129, 161, 200, 257, 300, 545, 1030):
        q, scale = lin.rows(T)
        lin.check(q, scale, lin.run(q, scale))


@pytest.mark.parametrize("T,K,N", [(2500, 512, 4096), (3000, 1024, 2048), (1500, 256, 16384), (4000, 256, 512)])
def test_linear_many_rows(T, K, N):
    lin = Linear(K, N, 65536)
    q, scale = lin.rows(T)
    lin.check(q, scale, lin.run(q, scale))


def test_linear_longest_sums():
    """All operands at the ends of their range, at the longest row that is taken: sums of -128 * -128 * 130816 stay below 2^31."""
    K, N = 130816, 128
    lin = Linear(K, N, 65536)
    lin.W.fill_(-128)
    lin.W[1] = 127
    host = torch.zeros_like(lin.pool, device="cpu")
    M.linear_pack(M.make_linear_shape(1, K, N, 65536, "i8"), lin.W, lin.table, host)
    lin.pool = host.cuda()
    for T in (1, 40, 300):
        q = torch.full((T, K), -128, dtype=torch.int8)
        q[T // 2] = 127
        scale = torch.full((T,), 2.0 ** -12)
        lin.check(q, scale, lin.run(q, scale))


@pytest.mark.parametrize("T", [1, 40, 100, 300, 700, 2500])
def test_linear_rows_are_their_own(T):
    """A row has the same bits in any call; a scale of NaN makes its row NaN and no other."""
    lin = Linear(512, 2176, 65536)
    q, scale = lin.rows(2500, seed=3)
    whole = lin.run(q, scale)
    scale2 = scale.clone()
    scale2[T // 2] = NAN
    part = lin.run(q[:T], scale2[:T])
    keep = torch.arange(T) != T // 2
    assert torch.equal(part.cpu()[keep], whole.cpu()[:T][keep]) and torch.isnan(part[T // 2]).all()


@pytest.mark.parametrize("T", [3, 50, 200, 2500])
def test_linear_bad_pages(T):
    """Entries outside the pool are read as page 0 and reported; the other column tiles are as they were."""
    lin = Linear(256, 2048, 16384)               # two pages to a column tile
    q, scale = lin.rows(T)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    lin.check(q, scale, lin.run(q, scale, status=status))
    assert status[0] == 0
    for entry, bad in ((0, -1), (31, lin.pool.shape[0]), (13, 2 ** 31 - 1)):
        table = lin.dev_table
        lin.dev_table = table.clone()
        lin.dev_table[entry] = bad
        out = lin.run(q, scale, status=status).cpu()
        lin.dev_table = table
        assert status[0].item() & 1
        want = O.product(q.numpy(), scale.numpy(), lin.W.numpy(), lin.w_scale.numpy())
        keep = np.arange(2048) // 128 != entry // 2
        assert (np.abs(out.numpy() - want) <= np.abs(want) * O.PRODUCT)[:, keep].all() and torch.isfinite(out).all()
        status.zero_()


# ---------------------------------------------------------------------------- the experts

class Experts:
    def __init__(self, H, F, E, k, page=16384, seed=0):
        g = torch.Generator().manual_seed(seed + H + F)
        self.H, self.F, self.E, self.k, self.page, self.g = H, F, E, k, page, g
        self.W = [torch.randint(-127, 128, shape, dtype=torch.int8, generator=g) for shape in ((E, F, H), (E, F, H), (E, H, F))]
        # gate and up values of a few units, so that both sides of the sigmoid and its middle are met
        about = 3.0 / (73.0 * 73.0 * H ** 0.5 * 0.02)
        self.scales = [torch.rand(shape, generator=g) * about + about / 2 for shape in ((E, F), (E, F))] + [torch.rand((E, H), generator=g) * 1e-3 + 5e-4]
        pw = M.PagedWeights(self.shape(1), *self.W, order=g, extra_pages=3).to_device()
        self.pool, self.table = pw.pages_dev, pw.table_dev
        self.dev = M.ExpertScales(*(s.cuda() for s in self.scales))

    def shape(self, T):
        return M.make_shape(T, self.H, self.F, self.E, self.k, "i8", self.page)

    def rows(self, T):
        return torch.randint(-127, 128, (T, self.H), dtype=torch.int8, generator=self.g), torch.rand(T, generator=self.g) * 0.02 + 0.01

    def routing(self, T, ids=None):
        """offsets, row_src, row_w of a routing: ids [T, k], or random with uneven experts."""
        if ids is None:
            logits = torch.randn((T, self.E), generator=self.g)
            logits[:, 0] += 1.5
            ids = logits.topk(self.k, dim=1).indices
        flat = ids.flatten()
        row_src = torch.sort(flat, stable=True).indices.to(torch.int32)
        counts = torch.bincount(flat, minlength=self.E)
        offsets = torch.cat([torch.zeros(1, dtype=torch.int64), counts.cumsum(0)]).to(torch.int32)
        return offsets, row_src, torch.rand(flat.numel(), generator=self.g)[row_src.long()] + 0.1

    def run(self, T, q, scale, offsets, row_src, row_w, **kw):
        return M.moe_expert_ffn_i8(self.shape(T), q.cuda(), scale.cuda(), offsets.cuda(), self.table, self.pool, self.dev, row_src=None if row_src is None else row_src.cuda(),
                                   row_w=None if row_w is None else row_w.cuda(), **kw)

    def check(self, q, scale, offsets, row_src, row_w, got, some=None):
        """some: at most so many rows of an expert are compared, its first, last and others between."""
        h_q, h_scale, out = (t.cpu().numpy() if t.dtype != torch.bfloat16 else bf16_values(t.cpu()) for t in got)
        for e in range(self.E):
            a, b = int(offsets[e]), int(offsets[e + 1])
            if a == b:
                continue
            r = np.arange(a, b) if some is None else np.unique(np.linspace(a, b - 1, some).round().astype(int))
            token = r if row_src is None else row_src.numpy()[r] // self.k
            W1, W3, W2 = (w[e].numpy() for w in self.W)
            s1, s3, s2 = (s[e].numpy() for s in self.scales)
            h, slack = O.gate_up(q.numpy()[token], scale.numpy()[token], W1, s1, W3, s3)
            slack = slack + (np.abs(h) + slack) * O.U16                       # h is rounded to bf16
            most, worst = np.abs(h).max(axis=1), slack.max(axis=1)
            step = h_scale[r].astype(np.float64)
            assert (np.abs(step * 127 - most) <= worst + most * 2 * O.U).all()
            assert (np.abs(h_q[r] * step[:, None] - h) <= slack + step[:, None] * (0.5 + 127 * 4 * O.U) + np.abs(h) * 2 * O.U).all()
            want = O.product(h_q[r], h_scale[r], W2, s2) * (1.0 if row_w is None else row_w.numpy()[r].astype(np.float64)[:, None])
            # the row weight one more product; then bf16
            assert (np.abs(out[r] - want) <= np.abs(want) * (O.U16 * 1.001 + 5 * O.U)).all(), e


SHAPES = {"tiny": (256, 512, 8, 2, 65536), "odd": (1280, 768, 5, 3, 16384 * 5), "small": (1024, 2816, 8, 2, 524288), "fine": (512, 256, 64, 8, 16384), "one": (512, 1280, 1, 1, 16384),
          "long": (256, 4352, 2, 1, 65536)}


@pytest.mark.parametrize("name", list(SHAPES))
def test_experts(name):
    x = Experts(*SHAPES[name])
    for T in (1, 2, 7, 16, 17, 40, 64, 129, 300, 601):
        q, scale = x.rows(T)
        offsets, row_src, row_w = x.routing(T)
        x.check(q, scale, offsets, row_src, row_w, x.run(T, q, scale, offsets, row_src, row_w), some=12)


@pytest.mark.parametrize("T", [1, 20, 200, 700, 1500])
def test_experts_permuted_rows_without_weights(T):
    """Rows that are given in the order of the experts, no row weights; every row is compared where there are few."""
    x = Experts(512, 768, 4, 2, 65536)
    offsets, row_src, _ = x.routing(T)
    q, scale = x.rows(T)
    token = row_src.long() // x.k
    got = x.run(T, q[token], scale[token], offsets, None, None)
    x.check(q[token], scale[token], offsets, None, None, got, some=None if T <= 200 else 40)
    through = x.run(T, q, scale, offsets, row_src, None)
    assert all(torch.equal(a, b) for a, b in zip(got, through))


@pytest.mark.parametrize("heights", [[0, 0, 513, 0], [256, 257, 272, 288], [289, 0, 1, 192], [31, 33, 63, 129], [544, 545, 160, 161], [1, 1, 1, 1], [0, 3, 0, 0], [300, 128, 900, 32]])
def test_experts_of_given_heights(heights):
    """Experts without rows, and row tiles at the heights where a block takes another loop."""
    x = Experts(256, 1280, 4, 1, 65536)
    ids = torch.cat([torch.full((n,), e) for e, n in enumerate(heights)])
    ids = ids[torch.randperm(len(ids), generator=torch.Generator().manual_seed(5))][:, None]
    T = len(ids)
    q, scale = x.rows(T)
    offsets, row_src, row_w = x.routing(T, ids)
    x.check(q, scale, offsets, row_src, row_w, x.run(T, q, scale, offsets, row_src, row_w))


@pytest.mark.parametrize("T", [3, 60, 400, 1200])
def test_experts_rows_are_their_own(T):
    """A token's row has the same bits whatever the others hold; a scale of NaN makes its rows NaN and no others."""
    x = Experts(512, 1024, 4, 2, 65536)
    q, scale = x.rows(T)
    offsets, row_src, row_w = x.routing(T)
    first = x.run(T, q, scale, offsets, row_src, row_w)
    scale2, q2 = scale.clone(), q.clone()
    bad = T // 2
    scale2[bad] = NAN
    h_q, h_scale, out = (t.cpu() for t in x.run(T, q2, scale2, offsets, row_src, row_w))
    of_bad = (row_src.long() // x.k) == bad
    assert torch.isnan(h_scale[of_bad]).all() and torch.isnan(out[of_bad]).all() and (h_q[of_bad] == 0).all()
    for a, b in zip(first, (h_q, h_scale, out)):
        assert torch.equal(a.cpu()[~of_bad], b[~of_bad])
    q3 = torch.randint(-127, 128, q.shape, dtype=torch.int8)
    q3[bad] = q[bad]
    for a, b in zip(first, x.run(T, q3, scale, offsets, row_src, row_w)):
        assert torch.equal(a.cpu()[of_bad], b.cpu()[of_bad])


@pytest.mark.parametrize("H,F,E", [(512, 1024, 2), (256, 2816, 8), (256, 14336, 8), (2048, 512, 8)])
def test_experts_rows_have_the_same_bits_in_every_kernel(H, F, E):
    """Up to 2, 30, 75 and up to 1000 rows per expert on average are the kernels for a handful of tokens, for few rows (64 and 128, in blocks of 64, 112 and 128 features and of
    32, 64 and 128 columns by the size), and blocks of 256 rows (halved, narrow)."""
    x = Experts(H, F, E, 1, 65536)
    q, scale = x.rows(1000 * E)
    ids = torch.randint(0, E, (1000 * E, 1), generator=x.g)
    ids[:3] = torch.tensor([[0], [1], [0]])
    first = None
    for T in (3, 30 * E, 60 * E, 75 * E, 150 * E, 450 * E, 1000 * E):
        offsets, row_src, _ = x.routing(T, ids[:T])
        got = x.run(T, q[:T], scale[:T], offsets, row_src, None)
        at = [int((row_src == t).nonzero()) for t in range(3)]
        mine = [t.cpu()[at] for t in got]
        first = first or mine
        assert all(torch.equal(a, b) for a, b in zip(first, mine)), T


@pytest.mark.parametrize("T", [4, 100, 900])
def test_experts_bad_pages(T):
    x = Experts(256, 512, 4, 2, 16384)
    q, scale = x.rows(T)
    offsets, row_src, row_w = x.routing(T)
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    want = x.run(T, q, scale, offsets, row_src, row_w, status=status)
    assert status[0] == 0
    e = int(torch.bincount(torch.repeat_interleave(torch.arange(4), (offsets[1:] - offsets[:-1]).long()), minlength=4).argmax())
    other = torch.ones(row_src.numel(), dtype=torch.bool)
    other[int(offsets[e]):int(offsets[e + 1])] = False
    for entry, bad in ((0, -1), (x.table.shape[1] - 1, x.pool.shape[0])):
        table = x.table
        x.table = table.clone()
        x.table[e, entry] = bad
        got = x.run(T, q, scale, offsets, row_src, row_w, status=status)
        x.table = table
        assert status[0].item() & 1
        assert all(torch.equal(a.cpu()[other], b.cpu()[other]) for a, b in zip(want, got))
        status.zero_()


def test_experts_rows_behind_the_last_expert_stay():
    """offsets that end before R: the rows behind are neither computed nor written."""
    x = Experts(512, 1024, 4, 2, 65536)
    lib = B._lib()
    for T in (5, 100, 900):
        q, scale = x.rows(T)
        offsets, row_src, row_w = x.routing(T)
        cut = int(offsets[3])                    # the last expert has no rows now
        offsets[4] = cut
        R = 2 * T
        dev = [t.cuda() for t in (q, scale, row_src, offsets, row_w)]
        h_q, h_scale = torch.full((R, 1024), 77, dtype=torch.int8, device="cuda"), torch.full((R,), 5.0, device="cuda")
        h, out = torch.full((R, 1024), NAN, dtype=torch.bfloat16, device="cuda"), torch.full((R, 512), 9.0, dtype=torch.bfloat16, device="cuda")
        s = x.shape(T)
        rc = lib.moe_expert_ffn_i8(B.ctypes.byref(s), dev[0].data_ptr(), dev[1].data_ptr(), dev[2].data_ptr(), dev[3].data_ptr(), x.table.data_ptr(), x.pool.data_ptr(), x.pool.shape[0],
                                   x.dev.pointers(s), dev[4].data_ptr(), h.data_ptr(), h_q.data_ptr(), h_scale.data_ptr(), out.data_ptr(), None, B._stream(None))
        assert rc == 0
        assert (h_q[cut:] == 77).all() and (h_scale[cut:] == 5).all() and (out[cut:] == 9).all() and torch.isnan(h[cut:]).all()
        x.check(q, scale, offsets, row_src, row_w, (h_q, h_scale, out), some=10)


def test_experts_intermediates_beyond_32_bits():
    """h of more than 2^32 bytes, h_q of more than 2^31: the last rows are as right as the first."""
    T, x = 152000, Experts(256, 14336, 2, 1, 65536)
    q, scale = x.rows(T)
    ids = (torch.arange(T) >= T - 300).long()[:, None]
    offsets, row_src, row_w = x.routing(T, ids)
    assert T * 14336 > 2 ** 31
    h_q, h_scale, out = x.run(T, q, scale, offsets, row_src, row_w)
    rows = torch.tensor([0, 1, 70000, 149000, T - 301, T - 300, T - 256, T - 1])
    few = torch.tensor([0, 5, 8], dtype=torch.int32)
    got = [t[rows.cuda()] for t in (h_q, h_scale, out)]
    token = row_src[rows].long()
    x.check(q[token], scale[token], few, None, row_w[rows], got)


@pytest.mark.parametrize("option", ["xcd_remap", "half_tiles", "tall_tiles", "tall_first", "chunked", "balance", "down_cols"])
def test_options_change_no_bit(option):
    x = Experts(256, 1280, 4, 1, 65536)
    lin = Linear(256, 2176, 65536)
    rows = {T: (x.rows(T), x.routing(T)) for T in (40, 700, 1500)}
    lin_rows = lin.rows(1500)

    def all_of_it():
        return [t for T, (r, p) in rows.items() for t in x.run(T, *r, *p)] + [lin.run(*lin_rows)]

    want, value = all_of_it(), M.get_option(option)
    try:
        for v in {"chunked": (0, 8), "down_cols": (1, 2)}.get(option, (0,)):
            M.set_option(option, v)
            assert all(torch.equal(a, b) for a, b in zip(want, all_of_it())), v
    finally:
        M.set_option(option, value)


def test_more_rows_than_blocks():
    """Rows beyond 2^20 blocks are taken in turn."""
    T = (1 << 20) + 77
    x = torch.randn((4 * T, 4), device="cuda")
    q, scale = M.moe_quantize_i8(x)
    rows = torch.tensor([0, 1, T - 1, 4 * (1 << 20) - 1, 4 * (1 << 20), 4 * (1 << 20) + 5, 4 * T - 1])
    check_quantized(x.cpu()[rows], q.cpu()[rows], scale.cpu()[rows])
    y = torch.randn((T, 520), device="cuda").to(torch.bfloat16)
    q, scale = M.moe_quantize_i8(y)
    rows = torch.tensor([0, T - 78, T - 77, T - 1])
    check_quantized(y[rows.cuda()].cpu(), q[rows.cuda()], scale[rows.cuda()])
    delta, gamma = torch.randn((T, 260), device="cuda"), torch.ones(260, device="cuda")
    got = M.moe_add_rmsnorm_i8(None, delta, gamma, 1e-5)
    check_norm(None, delta[rows.cuda()].cpu(), gamma.cpu(), 1e-5, [t[rows.cuda()] for t in got])


# ---------------------------------------------------------------------------- together

def layer_inputs(T, H=512, F=768, E=4, k=2, seed=0, K=None):
    x = Experts(H, F, E, k, 65536, seed=seed)
    g = torch.Generator().manual_seed(seed + T)
    delta, gamma = torch.randn((T, H), generator=g), 1 + 0.1 * torch.randn(H, generator=g)
    Wr = (torch.randn((E, H), generator=g) * 0.1).to(torch.bfloat16)
    return x, delta.cuda(), gamma.cuda(), Wr.cuda()


@pytest.mark.parametrize("T", [1, 5, 40, 300, 1100])
def test_layer_is_its_parts(T):
    """moe_layer_i8 gives the bits of its calls made one after another."""
    x, delta, gamma, Wr = layer_inputs(T)
    _, rows, q, scale = M.moe_add_rmsnorm_i8(None, delta, gamma, 1e-5)
    s = x.shape(T)
    bias = torch.tensor([0.3, -0.2, 0.0, 0.1]).cuda()
    y, ws = M.moe_layer_i8(s, rows, q, scale, Wr, x.table, x.pool, x.dev, bias=bias)
    assert ws[:4].view(torch.int32).item() == 0
    ids, w, _ = M.moe_route(s.routed(), rows, Wr, bias)
    p = M.moe_permute(s.routed(), ids, topk_w=w)
    _, _, out = M.moe_expert_ffn_i8(s, q, scale, p["offsets"], x.table, x.pool, x.dev, row_src=p["row_src"], row_w=p["row_w"])
    assert torch.equal(y, M.moe_combine(s, out, p["row_of"]))
    picked = out.float()[p["row_of"].view(T, 2).long()]
    assert torch.equal(y, picked[:, 0] + picked[:, 1])


@pytest.mark.parametrize("T", [1, 17, 300])
def test_tasks_are_their_parts(T):
    """moe_pre_attention_i8 and moe_post_attention_i8 give the bits of their calls made one after another."""
    H, K = 512, 768
    x, delta, gamma, Wr = layer_inputs(T, seed=3)
    lin, o = Linear(H, 1024, 65536), Linear(K, H, 65536)
    g = torch.Generator().manual_seed(T)
    hidden, attn = torch.randn((T, H), generator=g).cuda(), torch.randn((T, K), generator=g).to(torch.bfloat16).cuda()
    ls = M.make_linear_shape(T, H, 1024, 65536, "i8")
    status = torch.zeros(4, dtype=torch.int32, device="cuda")
    got = M.moe_pre_attention_i8(ls, hidden, delta, gamma, 1e-5, lin.dev_table, lin.pool, lin.dev_scale, status=status)
    hs, _, q, scale = M.moe_add_rmsnorm_i8(hidden, delta, gamma, 1e-5, want_x=False)
    for a, b in zip(got, (hs, q, scale, M.moe_linear_i8(ls, q, scale, lin.dev_table, lin.pool, lin.dev_scale))):
        assert torch.equal(a, b)
    # one pool for the O projection and the experts
    pool = torch.cat([x.pool, o.pool])
    o_table = o.dev_table + x.pool.shape[0]
    s, os = x.shape(T), M.make_linear_shape(T, K, H, 65536, "i8")
    mid, x_moe, y, _ = M.moe_post_attention_i8(s, os, attn, hidden, o_table, o.dev_scale, gamma, 1e-5, Wr, x.table, pool, x.dev)
    a_q, a_scale = M.moe_quantize_i8(attn)
    proj = M.moe_linear_i8(os, a_q, a_scale, o_table, pool, o.dev_scale)
    hs, rows, q, scale = M.moe_add_rmsnorm_i8(hidden, proj, gamma, 1e-5)
    want, _ = M.moe_layer_i8(s, rows, q, scale, Wr, x.table, pool, x.dev)
    assert torch.equal(mid, hs) and torch.equal(x_moe, rows) and torch.equal(y, want)


def test_no_tokens():
    """T = 0 does nothing and returns empty arrays."""
    x = Experts(256, 512, 4, 2)
    s = x.shape(0)
    z = dict(device="cuda")
    q, scale = M.moe_quantize_i8(torch.empty((0, 256), **z))
    assert q.shape == (0, 256) and scale.shape == (0,)
    hs, rows, q, scale = M.moe_add_rmsnorm_i8(None, torch.empty((0, 256), **z), torch.ones(256, **z), 1e-5)
    lin = Linear(256, 128)
    assert M.moe_linear_i8(M.make_linear_shape(0, 256, 128, 16384, "i8"), q, scale, lin.dev_table, lin.pool, lin.dev_scale).shape == (0, 128)
    e = torch.zeros(5, dtype=torch.int32, **z)
    assert M.moe_expert_ffn_i8(s, q, scale, e, x.table, x.pool, x.dev)[2].shape == (0, 256)
    assert M.moe_layer_i8(s, rows, q, scale, torch.zeros((4, 256), dtype=torch.bfloat16, **z), x.table, x.pool, x.dev)[0].shape == (0, 256)


def test_two_layers_at_once():
    """Two calls on two streams, each with its own workspace and both on the same weights, many times over each other."""
    x, delta, gamma, Wr = layer_inputs(700, seed=5)
    s = x.shape(700)
    inputs = [M.moe_add_rmsnorm_i8(None, delta * f, gamma, 1e-5)[1:] for f in (1.0, -0.5)]
    want = [M.moe_layer_i8(s, *i, Wr, x.table, x.pool, x.dev)[0].clone() for i in inputs]
    streams = [torch.cuda.Stream() for _ in inputs]
    spaces = [torch.empty(M.layer_i8_workspace_bytes(s), dtype=torch.uint8, device="cuda") for _ in inputs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(10):
        for n, st in enumerate(streams):
            got[n].append(M.moe_layer_i8(s, *inputs[n], Wr, x.table, x.pool, x.dev, workspace=spaces[n], stream=st)[0])
    torch.cuda.synchronize()
    assert all(torch.equal(y, w) for ys, w in zip(got, want) for y in ys)


def test_on_a_stream_of_its_own_and_in_a_graph():
    """The whole run, residual to layer, on another stream and captured; replays with new inputs between eager calls give the eager bits."""
    T = 70
    x, delta, gamma, Wr = layer_inputs(T, seed=7)
    s = x.shape(T)
    ws = torch.empty(M.layer_i8_workspace_bytes(s), dtype=torch.uint8, device="cuda")

    def run(d):
        _, rows, q, scale = M.moe_add_rmsnorm_i8(None, d, gamma, 1e-5)
        return M.moe_layer_i8(s, rows, q, scale, Wr, x.table, x.pool, x.dev, workspace=ws)[0]

    want = run(delta).clone()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = run(delta)
    side.synchronize()
    assert torch.equal(got, want)
    _, rows, q, scale = M.moe_add_rmsnorm_i8(None, delta, gamma, 1e-5, stream=side)
    y, _ = M.moe_layer_i8(s, rows, q, scale, Wr, x.table, x.pool, x.dev, stream=side)
    side.synchronize()
    assert torch.equal(y, want)
    static = delta.clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(static)
    for i in range(4):
        static.copy_(delta * (i + 1) - i)
        graph.replay()
        torch.cuda.synchronize()
        captured = out.clone()
        assert torch.equal(captured, run(delta * (i + 1) - i)), i
